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
  float eps = 0.f;
  // backward: sums of each workgroup [wgs][stride] (dweight, then dbias), joined
  float* part = nullptr;
  float* dweight = nullptr;
  float* dbias = nullptr;
  int32_t stride = 0;
};

struct DropoutArgs {
  RowTensor x, res, y;         // res may be null
  DropArgs drop;
  int32_t rows = 0, cols = 0;
  Divisor tokens, chunks;      // chunks: of a row
};

// What stands in front of a norm.
enum NormKind { NORM_ALONE = 0, NORM_RESIDUAL = 1, NORM_DROPOUT = 2 };

hipError_t launch_norm_fwd(const NormArgs& a, int dtype, NormKind kind, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs& a, int dtype, NormKind kind, hipStream_t s);
// Workgroups of the backward for this many rows, and floats of each one's sums.
int norm_bwd_wgs(int64_t rows, int cols);
inline int norm_part_stride(int cols) { return (2 * cols + 63) / 64 * 64; }
hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s);

#ifdef __HIPCC__

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// (the loads and stores below are single 16-byte ones at any alignment of the
// element: global memory is accessed unaligned on this target)
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));

// Eight elements as they are stored.
template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> {
  u32x4 r;
  __device__ __forceinline__ void clear() { r = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const bf16_t* p) {
    r = *reinterpret_cast<const u32x4_at2*>(p);
  }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<u32x4_at2*>(p) = r; }
  __device__ __forceinline__ float get(int e) const {
    return __uint_as_float(e % 2 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = uint32_t(f2bf(v[2 * k])) | uint32_t(f2bf(v[2 * k + 1])) << 16;
  }
  __device__ __forceinline__ void put(int e, bf16_t x) {
    r[e / 2] = e % 2 ? (r[e / 2] & 0xffffu) | uint32_t(x) << 16 : (r[e / 2] & 0xffff0000u) | x;
  }
  __device__ __forceinline__ bf16_t at(int e) const { return bf16_t(r[e / 2] >> (e % 2 * 16)); }
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
  __device__ __forceinline__ float get(int e) const { return __uint_as_float(r[e / 4][e % 4]); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e / 4][e % 4] = __float_as_uint(v[e]);
  }
  __device__ __forceinline__ void put(int e, float x) { r[e / 4][e % 4] = __float_as_uint(x); }
  __device__ __forceinline__ float at(int e) const { return get(e); }
};

// The chunk at p, of which m elements are in the row (at most 0: none).
template <typename T>
__device__ __forceinline__ void load_chunk(Chunk<T>& c, const T* p, int m) {
  if (m >= 8) {
    c.load(p);
    return;
  }
  c.clear();
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < m) c.put(e, p[e]);
}
template <typename T>
__device__ __forceinline__ void store_chunk(const Chunk<T>& c, T* p, int m) {
  if (m >= 8) {
    c.store(p);
    return;
  }
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < m) p[e] = c.at(e);
}

// Where a row lies: its tensor's start plus (sequence, token).
struct RowAt {
  uint32_t b, t;
};
template <typename T>
__device__ __forceinline__ T* row_of(const RowTensor& x, RowAt at) {
  return reinterpret_cast<T*>(x.p + int64_t(at.b) * x.b + int64_t(at.t) * x.t);
}

// v of the elements that stay, scaled; 0 of the others, whatever they hold. (No
// fused multiply-add with what follows: the sum with a residual has the same bits
// wherever it is formed.)
__device__ __forceinline__ void drop(float (&v)[8], const DropArgs& d, uint64_t seed, uint64_t offset,
                                     uint32_t row, uint32_t chunk) {
#pragma clang fp contract(off)
  const Philox u = dropout_draws(seed, offset, d.site, row, chunk);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t draw = e % 2 ? u.w[e / 2] >> 16 : u.w[e / 2] & 0xffffu;
    v[e] = draw < d.threshold ? 0.f : v[e] * d.scale;
  }
}

__device__ __forceinline__ float plain_add(float x, float y) {
#pragma clang fp contract(off)
  return x + y;
}

// Sums of two values over the LPR lanes that share a row (a power of two from 8;
// above 64 the workgroup is the row, and `turn` alternates between two places of
// the exchange: one barrier a sum). Every lane has the same bits.
template <int LPR>
__device__ __forceinline__ float2 row_sum(float2 v, float2* sh, int& turn) {
  constexpr int W = LPR < 64 ? LPR : 64;
  v.x = group_sum<W>(v.x);
  v.y = group_sum<W>(v.y);
  if constexpr (LPR > 64) {
    constexpr int N = LPR / 64;
    float2* at = sh + turn * N;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int k = 1; k < N; ++k) {
      v.x += at[k].x;
      v.y += at[k].y;
    }
  }
  return v;
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

// Lanes that share a row, and chunks each of them holds.
template <int LPR_, int NV_> struct NormShape {
  static constexpr int LPR = LPR_, NV = NV_;
  static constexpr int NT = LPR > 64 ? LPR : 256;  // threads of a workgroup
  static constexpr int R = NT / LPR;                // rows it holds at a time
};

// f(shape) for the smallest shape that holds `chunks` chunks a row.
template <typename F> auto with_shape(int chunks, F f) {
  if (chunks <= 8) return f(NormShape<8, 1>());
  if (chunks <= 16) return f(NormShape<16, 1>());
  if (chunks <= 32) return f(NormShape<32, 1>());
  if (chunks <= 64) return f(NormShape<64, 1>());
  if (chunks <= 96) return f(NormShape<32, 3>());
  if (chunks <= 128) return f(NormShape<64, 2>());
  if (chunks <= 256) return f(NormShape<128, 2>());
  if (chunks <= 512) return f(NormShape<256, 2>());
  if (chunks <= 1024) return f(NormShape<512, 2>());
  return f(NormShape<1024, 2>());
}

#endif  // __HIPCC__

}  // namespace abft
