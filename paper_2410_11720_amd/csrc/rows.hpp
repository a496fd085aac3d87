// Rows of a [batch, tokens, cols] tensor in chunks of eight elements: loads and
// stores at any alignment, sums over the lanes that share a row. Included by the
// kernels of layer norm and dropout; RowTensor and the arguments by the entry
// points too.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "abft_device.hpp"
#include "abft_internal.hpp"
#include "divide.hpp"
#include "philox.hpp"

namespace abft {

struct RowTensor {
  char* p = nullptr;
  int64_t b = 0, t = 0;  // bytes between sequences, between tokens
};

// Dropout's part of a kernel's arguments: an element stays if its 16-bit draw is
// not below the threshold, and is scaled.
struct DropArgs {
  const uint64_t* rng = nullptr;  // seed, offset
  uint32_t threshold = 0, site = 0;
  uint32_t last = 0;              // (threshold << 16) - 1
  float scale = 1.f;
};

struct NormArgs {
  RowTensor x, res, h, y;      // forward: h may be null; backward reads h
  RowTensor dy, dh, dx, dres;  // backward: dh, dx and dres may be null
  const void* weight = nullptr;
  const void* bias = nullptr;
  int weight_bf16 = 0;
  const int32_t* lens = nullptr;
  float2* stats = nullptr;     // mean, 1 / deviation of each row; forward: may be null
  DropArgs drop;
  int32_t rows = 0, cols = 0;
  Divisor tokens;
  float eps = 0.f, eps_scaled = 0.f;  // the second: of a row scaled by 2^-80
  // backward: sums of each workgroup [wgs][stride] (dweight, then dbias), joined
  float* part = nullptr;
  float* dweight = nullptr;
  float* dbias = nullptr;
  int32_t stride = 0;
  int32_t mode = 0;            // ROWS_...
};

// How rows lie: of whole chunks at multiples of 16 bytes; of at least a chunk at
// multiples of 4; any other. For the first two, tensors of rows below a wave's width are
// below 2 GiB, and statistics too.
enum RowMode { ROWS_ANY = 0, ROWS_CHUNKS = 1, ROWS_WORDS = 2 };

struct DropoutArgs {
  RowTensor x, res, y;         // res may be null
  DropArgs drop;
  int32_t rows = 0, cols = 0;
  Divisor tokens, chunks;      // chunks: of a row
  int32_t flat = 0;            // all tensors are whole chunks, one behind the other, at
                               // multiples of 16 bytes
};

// Columns up to which less than a wave shares a row of whole chunks.
constexpr int NORM_LINE_COLS = 768;

// What stands in front of a norm.
enum NormKind { NORM_ALONE = 0, NORM_RESIDUAL = 1, NORM_DROPOUT = 2 };

hipError_t launch_norm_fwd(const NormArgs& a, int dtype, NormKind kind, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs& a, int dtype, NormKind kind, hipStream_t s);
// Workgroups of the backward for this many rows, and floats of each one's sums.
int norm_bwd_wgs(int64_t rows, int cols);
// (each sum's columns rounded up to whole chunks, both to whole joining workgroups)
__host__ __device__ inline int norm_padded(int cols) { return (cols + 7) / 8 * 8; }
inline int norm_part_stride(int cols) { return (2 * norm_padded(cols) + 31) / 32 * 32; }
hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s);

#ifdef __HIPCC__

// A launch without the configuration's detour through the runtime (2.2 instead of 2.5
// us, of calls that take 8).
template <typename... A>
hipError_t start(void (*kernel)(A...), dim3 grid, int threads, size_t lds, hipStream_t s, A... args) {
  void* at[] = {&args...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, lds, s);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// (the loads and stores below are single 16-byte ones at any alignment of the
// element: global memory is accessed unaligned on this target)
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
typedef u32x2 u32x2_at4 __attribute__((aligned(4)));
typedef uint32_t u32_at2 __attribute__((aligned(2)));

// Eight elements as they are stored.
template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> {
  u32x4 r;
  __device__ __forceinline__ void clear() { r = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const bf16_t* p) {
    r = *reinterpret_cast<const u32x4_at2*>(p);
  }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<u32x4_at2*>(p) = r; }
  __device__ __forceinline__ void store_past(bf16_t* p) const {  // past the cache, aligned
    __builtin_nontemporal_store(r, reinterpret_cast<u32x4*>(p));
  }
  __device__ __forceinline__ float get(int e) const {
    return __uint_as_float(e % 2 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // (two in one conversion)
      const f32x2 f = {v[2 * k], v[2 * k + 1]};
      r[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
    }
  }
  __device__ __forceinline__ void put(int e, bf16_t x) {
    r[e / 2] = e % 2 ? (r[e / 2] & 0xffffu) | uint32_t(x) << 16 : (r[e / 2] & 0xffff0000u) | x;
  }
  __device__ __forceinline__ void keep(bool yes) {  // else all 0
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = yes ? r[k] : 0;
  }
  // What is computed from it anew is not kept from before.
  __device__ __forceinline__ void anew() {
#pragma unroll
    for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(r[k]));
  }
  __device__ __forceinline__ void down(int n) {  // element e + n to e, 0 behind; n in 0 .. 7
    u32x4 t = n & 4 ? u32x4{r[2], r[3], 0, 0} : r;
    t = n & 2 ? u32x4{t[1], t[2], t[3], 0} : t;
    const u32x4 next = {t[1], t[2], t[3], 0};
    r = n & 1 ? t >> 16 | next << 16 : t;
  }
  // its first 4, 2 or 1 elements
  __device__ __forceinline__ void store4(bf16_t* p) const {
    *reinterpret_cast<u32x2_at2*>(p) = u32x2{r[0], r[1]};
  }
  __device__ __forceinline__ void store2(bf16_t* p) const { *reinterpret_cast<u32_at2*>(p) = r[0]; }
  __device__ __forceinline__ void store1(bf16_t* p) const { *p = bf16_t(r[0]); }
};
template <> struct Chunk<float> {
  u32x4 r[2];
  __device__ __forceinline__ void clear() { r[0] = r[1] = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const float* p) {
    r[0] = reinterpret_cast<const u32x4_at4*>(p)[0];
    r[1] = reinterpret_cast<const u32x4_at4*>(p)[1];
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<u32x4_at4*>(p)[0] = r[0];
    reinterpret_cast<u32x4_at4*>(p)[1] = r[1];
  }
  __device__ __forceinline__ void store_past(float* p) const {
    __builtin_nontemporal_store(r[0], reinterpret_cast<u32x4*>(p));
    __builtin_nontemporal_store(r[1], reinterpret_cast<u32x4*>(p) + 1);
  }
  __device__ __forceinline__ float get(int e) const { return __uint_as_float(r[e / 4][e % 4]); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e / 4][e % 4] = __float_as_uint(v[e]);
  }
  __device__ __forceinline__ void put(int e, float x) { r[e / 4][e % 4] = __float_as_uint(x); }
  __device__ __forceinline__ void keep(bool yes) {
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k / 4][k % 4] = yes ? r[k / 4][k % 4] : 0;
  }
  __device__ __forceinline__ void anew() {
#pragma unroll
    for (int k = 0; k < 8; ++k) asm volatile("" : "+v"(r[k / 4][k % 4]));
  }
  __device__ __forceinline__ void down(int n) {
    const u32x4 z = {0, 0, 0, 0};
    u32x4 a = n & 4 ? r[1] : r[0], b = n & 4 ? z : r[1];
    a = n & 2 ? u32x4{a[2], a[3], b[0], b[1]} : a;
    b = n & 2 ? u32x4{b[2], b[3], 0, 0} : b;
    r[0] = n & 1 ? u32x4{a[1], a[2], a[3], b[0]} : a;
    r[1] = n & 1 ? u32x4{b[1], b[2], b[3], 0} : b;
  }
  __device__ __forceinline__ void store4(float* p) const { *reinterpret_cast<u32x4_at4*>(p) = r[0]; }
  __device__ __forceinline__ void store2(float* p) const {
    *reinterpret_cast<u32x2_at4*>(p) = u32x2{r[0][0], r[0][1]};
  }
  __device__ __forceinline__ void store1(float* p) const { *p = __uint_as_float(r[0][0]); }
};

// The chunk at p, of which m elements are in the row (at most 0: none). The loads of a
// part are all in flight at once (the last element's in the place of those behind it).
template <typename T>
__device__ __forceinline__ void load_chunk(Chunk<T>& c, const T* p, int m) {
  if (m >= 8) {
    c.load(p);
    return;
  }
  c.clear();
  if (m <= 0) return;
  T t[7];
#pragma unroll
  for (int e = 0; e < 7; ++e) t[e] = p[min(e, m - 1)];
#pragma unroll
  for (int e = 0; e < 7; ++e) c.put(e, e < m ? t[e] : T(0));
}
template <typename T>
__device__ __forceinline__ void store_chunk(Chunk<T> c, T* p, int m) {
  if (m >= 8) {
    c.store(p);
    return;
  }
  if (m <= 0) return;
  if (m & 4) {
    c.store4(p);
    c.down(4);
    p += 4;
  }
  if (m & 2) {
    c.store2(p);
    c.down(2);
    p += 2;
  }
  if (m & 1) c.store1(p);
}

// Where a row lies: its tensor's start plus (sequence, token).
struct RowAt {
  uint32_t b, t;
};
__device__ __forceinline__ RowAt row_at(const Divisor& tokens, uint32_t row) {
  RowAt at;
  at.b = tokens.quotient(row);
  at.t = row - at.b * tokens.d;
  return at;
}
template <typename T>
__device__ __forceinline__ T* row_of(const RowTensor& x, RowAt at) {
  return reinterpret_cast<T*>(x.p + int64_t(at.b) * x.b + int64_t(at.t) * x.t);
}

// v of the elements that stay, scaled; 0 of the others, whatever they hold. (No
// fused multiply-add with what follows: the sum with a residual has the same bits
// wherever it is formed.) The draws are compared in the high halves of words: one is
// below t exactly if the word is at most (t << 16) - 1.
__device__ __forceinline__ void drop(float (&v)[8], const DropArgs& d, uint64_t seed, uint64_t offset,
                                     uint32_t row, uint32_t chunk) {
#pragma clang fp contract(off)
  const Philox u = dropout_draws(seed, offset, d.site, row, chunk);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t word = e % 2 ? u.w[e / 2] : u.w[e / 2] << 16;
    v[e] = word <= d.last ? 0.f : v[e] * d.scale;
  }
}

__device__ __forceinline__ float plain_add(float x, float y) {
#pragma clang fp contract(off)
  return x + y;
}

// Sum over aligned groups of W lanes (a power of two from 8), in every lane of a
// group: lane moves within 16, swaps of 16 and 32 lanes.
template <int W> __device__ __forceinline__ float lanes_sum(float x) {
  x = group_sum<W < 16 ? W : 16>(x);
  if constexpr (W >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (W >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// A gain or offset's eight entries from column col on (m in range).
__device__ __forceinline__ void load_params(float (&v)[8], const void* p, int bf16, int col, int m,
                                            float absent) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = absent;
  if (p == nullptr || m <= 0) return;
  if (bf16) {
    Chunk<bf16_t> c;
    load_chunk(c, static_cast<const bf16_t*>(p) + col, m);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c.get(e);
  } else {
    Chunk<float> c;
    load_chunk(c, static_cast<const float*>(p) + col, m);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c.get(e);
  }
}

// ---- rows by their lanes -------------------------------------------------------------
// Rows at multiples of 4 bytes are read and written through buffer descriptors, which
// bring 0 from outside of their bytes and drop what is stored there: a lane without a
// chunk, a row behind a sequence's length or behind the last one, a tensor that is not
// given need no branch. With branches around them the compiler cannot count what is in
// flight, and waits for the next row's loads and for all stores where it needs this
// row's (calls one after another, norm of 8192 x 768: forward 9.0 -> 7.3 us; 14500 x 1092
// with residual and dropout 52.4 -> 45.8). Rows of bf16 at odd elements take those
// branches. What lies where and the order of sums are the same, and so are the results' bits.
// Where less than a chunk is left of a row, its lane reads the row's last eight elements
// and `settle` moves what is its own to the front.

constexpr uint32_t OUTSIDE = 0x80000000u;  // an offset behind every descriptor's bytes

__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_at(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(bytes), 0x00020000);
}
__device__ __forceinline__ void load_at(Chunk<bf16_t>& c, __amdgpu_buffer_rsrc_t b, uint32_t off) {
  c.r = __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, 0);
}
__device__ __forceinline__ void load_at(Chunk<float>& c, __amdgpu_buffer_rsrc_t b, uint32_t off) {
  c.r[0] = __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, 0);
  c.r[1] = __builtin_amdgcn_raw_buffer_load_b128(b, off + 16, 0, 0);
}
__device__ __forceinline__ void store_at(const Chunk<bf16_t>& c, __amdgpu_buffer_rsrc_t b,
                                         uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b128(c.r, b, off, 0, 0);
}
__device__ __forceinline__ void store_at(const Chunk<float>& c, __amdgpu_buffer_rsrc_t b,
                                         uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b128(c.r[0], b, off, 0, 0);
  __builtin_amdgcn_raw_buffer_store_b128(c.r[1], b, off + 16, 0, 0);
}

// its first 4, 2 or 1 elements
__device__ __forceinline__ void store4_at(const Chunk<bf16_t>& c, __amdgpu_buffer_rsrc_t b, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b64(u32x2{c.r[0], c.r[1]}, b, off, 0, 0);
}
__device__ __forceinline__ void store2_at(const Chunk<bf16_t>& c, __amdgpu_buffer_rsrc_t b, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b32(c.r[0], b, off, 0, 0);
}
__device__ __forceinline__ void store4_at(const Chunk<float>& c, __amdgpu_buffer_rsrc_t b, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b128(c.r[0], b, off, 0, 0);
}
__device__ __forceinline__ void store2_at(const Chunk<float>& c, __amdgpu_buffer_rsrc_t b, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b64(u32x2{c.r[0][0], c.r[0][1]}, b, off, 0, 0);
}
__device__ __forceinline__ void store1_at(const Chunk<float>& c, __amdgpu_buffer_rsrc_t b, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b32(c.r[0][0], b, off, 0, 0);
}

// Lanes that share a row and chunks each of them holds (chunk lane + j lanes): LPR
// lanes, or (LPR = 0) the workgroup's waves divided among its rows.
template <int LPR_, int NV_> struct Shape {
  static constexpr int LPR = LPR_, NV = NV_;
};
struct ShapeAt {        // what the host chose
  int lanes, rows;      // of a row; of a workgroup
  int threads() const { return lanes * rows; }
};

// A thread's place: its row of the workgroup's, its chunks in a row.
template <typename T, typename S> struct Place {
  int lanes, lane, slot, cols;
  uint32_t off[S::NV];  // of its chunks in a row, bytes

  __device__ __forceinline__ Place(int lanes_, int cols_) : cols(cols_) {
    lanes = S::LPR ? S::LPR : lanes_;
    if constexpr (S::LPR) {
      slot = threadIdx.x / S::LPR;
      lane = threadIdx.x % S::LPR;
    } else {
      slot = threadIdx.x / uint32_t(lanes);
      lane = threadIdx.x - slot * lanes;
    }
    if constexpr (S::LPR == 0 || S::LPR >= 64) slot = __builtin_amdgcn_readfirstlane(slot);
#pragma unroll
    for (int j = 0; j < S::NV; ++j) off[j] = col(j) < cols ? col(j) * uint32_t(sizeof(T)) : OUTSIDE;
  }
  __device__ __forceinline__ int col(int j) const { return 8 * (lane + j * lanes); }
  __device__ __forceinline__ bool has(int j) const { return off[j] != OUTSIDE; }
  __device__ __forceinline__ int left(int j) const { return cols - col(j); }
};

// A row of x (ok false: none of it). Rows of one wave or more have a descriptor of
// their own, of fewer lanes an offset in their tensor's (below 2 GiB).
template <typename T, typename S, int MODE> struct Line {
  static constexpr bool WAVES = S::LPR == 0 || S::LPR >= 64;
  __amdgpu_buffer_rsrc_t b;
  uint32_t row;

  __device__ __forceinline__ Line(const RowTensor& x, RowAt at, bool ok, int cols)
      : b(bytes_at(nullptr, 0)), row(0) {
    if constexpr (WAVES) {
      b = bytes_at(x.p + int64_t(at.b) * x.b + int64_t(at.t) * x.t,
                   ok && x.p ? cols * uint32_t(sizeof(T)) : 0);
    } else {
      b = bytes_at(x.p, x.p ? OUTSIDE - 32 : 0);
      row = ok ? at.b * uint32_t(x.b) + at.t * uint32_t(x.t) : OUTSIDE;
    }
  }
  __device__ __forceinline__ uint32_t at(uint32_t off) const {
    if constexpr (WAVES) return off;
    return off != OUTSIDE && row != OUTSIDE ? off + row : OUTSIDE;
  }
  __device__ __forceinline__ void load(Chunk<T>& c, const Place<T, S>& p, int j) const {
    uint32_t off = p.off[j];
    if constexpr (MODE == ROWS_WORDS)
      off = p.has(j) ? min(off, uint32_t(p.cols - 8) * uint32_t(sizeof(T))) : OUTSIDE;
    load_at(c, b, at(off));
  }
  __device__ __forceinline__ void store(const Chunk<T>& c, const Place<T, S>& p, int j) const {
    if constexpr (MODE == ROWS_CHUNKS) {
      store_at(c, b, at(p.off[j]));
    } else {
      const int m = p.left(j);
      uint32_t off = p.off[j];
      store_at(c, b, at(m >= 8 ? off : OUTSIDE));
      if (__all(m >= 8 || m <= 0)) return;
      // (four, two and one of the elements that are left, if these are)
      const bool part = m > 0 && m < 8;
      Chunk<T> t = c;
      store4_at(t, b, at(part && (m & 4) ? off : OUTSIDE));
      off += m & 4 ? 4 * sizeof(T) : 0;
      t.down(m & 4);
      store2_at(t, b, at(part && (m & 2) ? off : OUTSIDE));
      if constexpr (sizeof(T) == 4) {
        off += m & 2 ? 2 * sizeof(T) : 0;
        t.down(m & 2);
        store1_at(t, b, at(part && (m & 1) ? off : OUTSIDE));
      }
    }
  }
};
template <typename T, typename S> struct Line<T, S, ROWS_ANY> {
  T* row;

  __device__ __forceinline__ Line(const RowTensor& x, RowAt at, bool ok, int)
      : row(ok && x.p ? row_of<T>(x, at) : nullptr) {}
  __device__ __forceinline__ void load(Chunk<T>& c, const Place<T, S>& p, int j) const {
    const int m = row ? p.cols - p.col(j) : 0;
    if (p.cols < 8)
      load_chunk(c, row + p.col(j), m);
    else if (m > 0)
      c.load(row + p.col(j) + min(0, m - 8));
  }
  __device__ __forceinline__ void store(const Chunk<T>& c, const Place<T, S>& p, int j) const {
    store_chunk(c, row + p.col(j), row ? p.cols - p.col(j) : 0);
  }
};

// A chunk as Line::load left it, with 0 for what is not in the row.
template <int MODE, typename T, typename S>
__device__ __forceinline__ void settle(Chunk<T>& c, const Place<T, S>& p, int j, bool ok) {
  if constexpr (MODE != ROWS_CHUNKS) {
    const int m = p.left(j);
    if (!__all(m >= 8) && p.cols >= 8) c.down(max(0, min(8 - m, 7)));
    if constexpr (MODE == ROWS_ANY) c.keep(ok && m > 0);
  }
}

// Sums of two values over the lanes of a row. Rows of several waves exchange their
// waves' sums in LDS, in one of two places by turns (one barrier a sum, which all the
// workgroup's waves pass).
template <typename S>
__device__ __forceinline__ float2 line_sum(float2 v, float2 (*sh)[16], int waves, int slot, int& turn) {
  constexpr int W = S::LPR && S::LPR < 64 ? S::LPR : 64;
  v.x = lanes_sum<W>(v.x);
  v.y = lanes_sum<W>(v.y);
  if constexpr (S::LPR == 0) {
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 15;
    float2* at = sh[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[wave] = v;
    __syncthreads();
    v = l < waves ? at[slot * waves + l] : make_float2(0.f, 0.f);
    v.x = group_sum<16>(v.x);
    v.y = group_sum<16>(v.y);
  }
  return v;
}

#endif  // __HIPCC__

}  // namespace abft
