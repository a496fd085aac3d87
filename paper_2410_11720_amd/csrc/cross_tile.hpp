// Building blocks of the attention kernels over keys of another length
// (cross_fwd.hip, cross_bwd.hip): operand tiles in LDS, their products on
// the matrix cores, and the relative position bias.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "abft_device.hpp"
#include "cross_internal.hpp"
#include "direct_lds.hpp"

namespace abft {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float NEG_INF = -__builtin_inff();
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_hw(float x) { return __builtin_amdgcn_logf(x); }

// x combined with the value of lane l ^ 32.
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef float float2_t __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const float2_t f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}

// Keeps the loads before it in front of what follows.
template <bool ON>
__device__ __forceinline__ void issue_loads() {
  if constexpr (ON) __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// Keys of a sequence, and the position of its first query among them (values
// that the host cannot check are brought into range here).
__device__ __forceinline__ int seq_len(const CrossArgs& a, int b) {
  return a.k_lens ? clampi(a.k_lens[b], 0, a.Sk) : a.Sk;
}
__device__ __forceinline__ int seq_start(const CrossArgs& a, int b) {
  return a.q_start ? clampi(a.q_start[b], -(1 << 29), 1 << 29) : 0;
}

// x - bf16(x) (0 where that is not a number: x INF or NaN)
__device__ __forceinline__ float rounding_rest(float x) {
  const float r = x - bf2f(f2bf(x));
  return r == r ? r : 0.f;
}

// 4 bytes per lane from the buffer to LDS [lds, lds + 256) in lane order.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma4(const u32x4& rs, uint32_t lds, uint32_t voff, uint32_t soff) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :
               : "s"(lds), "v"(voff), "s"(rs), "s"(soff)
               : "memory", "m0");
#endif
}
#pragma clang diagnostic pop

// A tile of rows of D elements in LDS, row-major, 16-byte chunk c of row r at
// chunk c ^ swz(r). LDS serves 256 bytes, a run of 16 chunks, at a time: the 16
// rows that share a step of a 16-byte read of one chunk lie at 16 places of
// it in bf16, and so do the 4 rows x 4 chunks of a transposing read. (With the 8
// places that a swizzle of three bits reaches, half of all LDS cycles were
// conflicts. fp32 keeps to three bits: its products take 16 times as long as their
// reads, and longer periods cost registers.)
//
// Products (32 x 32 tiles, lane l: column l % 32, half = l / 32):
//  rows  C[32 rows x 32] += tile rows . B, B's column the lane's own vector of
//        D elements (RowFrag)
//  cols  C[D x 32] += tile^T . P over 32 rows, P the 32 x 32 result of a
//        `rows` product: register r of it holds row 8 (r / 4) + 4 half + r % 4,
//        and the transposed operand is read in that order of rows, so P goes
//        from one product to the next in registers.
template <typename T, int D>
struct CrossTile {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int ROWB = D * int(sizeof(T));  // bytes per row
  static constexpr int CPR = ROWB / 16;            // chunks per row
  static constexpr int RPR = 64 / CPR;             // rows per 1-KB run
  static constexpr int NV = (BF ? 16 : 8) / RPR;   // runs until the swizzle repeats
  static constexpr int NF = D / (BF ? 16 : 8);     // fragments of a row vector
  static constexpr int ND = D / 32;                // 32-row blocks of a transposed product

  __device__ static __forceinline__ int swz(int r) {
    if constexpr (!BF) return ((r & 3) << 1) | ((r >> 2) & 1);
    else if constexpr (CPR == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    else return ((r & 3) << 2) | ((r >> 2) & 3);
  }

  // the lane's share of a row vector: 16-byte chunks 2 f + half
  struct RowFrag {
    u32x4 f[NF];
  };
  __device__ static __forceinline__ void load_row(RowFrag& q, const char* row, int half) {
#pragma unroll
    for (int f = 0; f < NF; ++f)
      q.f[f] = *reinterpret_cast<const u32x4*>(row + (2 * f + half) * 16);
  }
  __device__ static __forceinline__ void zero_row(RowFrag& q) {
#pragma unroll
    for (int f = 0; f < NF; ++f) q.f[f] = u32x4{0u, 0u, 0u, 0u};
  }
  // this lane's part of the dot product of two row vectors
  __device__ static __forceinline__ float dot_row(const RowFrag& a, const RowFrag& b) {
    float s = 0.f;
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BF) {
          s = fmaf(__uint_as_float(a.f[f][e] << 16), __uint_as_float(b.f[f][e] << 16), s);
          s = fmaf(__uint_as_float(a.f[f][e] & 0xffff0000u),
                   __uint_as_float(b.f[f][e] & 0xffff0000u), s);
        } else {
          s = fmaf(__uint_as_float(a.f[f][e]), __uint_as_float(b.f[f][e]), s);
        }
      }
    return s;
  }

  // Copies ROWS rows starting at `src` (rows ldb bytes apart) to the image at
  // `lds`, split over NW waves. Rows from `left` on repeat row left - 1, so
  // nothing past a sequence's end is read: what they bring is masked or never
  // stored. Likewise rows in front of row `low`. left > low, left >= 1.
  template <int ROWS, int NW>
  __device__ static __forceinline__ void issue(const char* src, uint32_t ldb, int left,
                                               uint32_t lds, int wave, int lane, int low = 0) {
    constexpr int PW = ROWS / RPR / NW;  // runs of this wave
    static_assert(PW * RPR * NW == ROWS, "whole runs a wave");
    const u32x4 rs = rsrc_of(src, 0x7fffffffu);
    const int r = lane / CPR, pos = lane % CPR;
    if (left >= ROWS && low <= 0) {
#pragma unroll
      for (int j = 0; j < PW; ++j) {
        const int i = wave * PW + j;
        const int rr = (PW % NV == 0 ? j : i) * RPR + r;  // the row, modulo the swizzle's period
        const uint32_t vo = uint32_t(r) * ldb + uint32_t((pos ^ swz(rr)) << 4);
        dma16(rs, uni(lds + i * 1024), vo, uni(uint32_t(i * RPR) * ldb));
      }
    } else {
#pragma unroll
      for (int j = 0; j < PW; ++j) {
        const int i = wave * PW + j, row = i * RPR + r;
        const uint32_t vo =
            uint32_t(clampi(row, low, left - 1)) * ldb + uint32_t((pos ^ swz(row)) << 4);
        dma16(rs, uni(lds + i * 1024), vo, 0u);
      }
    }
  }

  // Fragments of 32 rows of an image as the first operand of a `rows` product.
  // Products are written as a load and a multiply, so that a kernel can issue
  // the loads of a product before the work in front of it: left to itself the
  // compiler reads every fragment right before its instruction and waits.
  __device__ static __forceinline__ void load_rows(RowFrag& a, const char* img, int row0,
                                                   int lane) {
    const int r = lane & 31, half = lane >> 5;
    const char* p = img + (row0 + r) * ROWB;
    const int sw = swz(r);
#pragma unroll
    for (int f = 0; f < NF; ++f)
      a.f[f] = *reinterpret_cast<const u32x4*>(p + (((2 * f + half) ^ sw) << 4));
  }
  // C += A B
  __device__ static __forceinline__ void rows(floatx16& c, const RowFrag& a, const RowFrag& b) {
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      if constexpr (BF) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.f[f]),
                                                    __builtin_bit_cast(bf16x8, b.f[f]), c, 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.f[f][e]),
                                                   __uint_as_float(b.f[f][e]), c, 0, 0, 0);
      }
    }
  }

  // C += (rows [row0, row0 + 32) of the image) B, B's columns the rows [at, at +
  // 32) of another image: fragment by fragment, for few registers.
  __device__ static __forceinline__ void rows(floatx16& c, const char* img, int row0,
                                              const char* own, int at, int lane) {
    const int r = lane & 31, half = lane >> 5;
    const char* p = img + (row0 + r) * ROWB;
    const char* q = own + (at + r) * ROWB;
    const int sw = swz(r);
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const int ch = ((2 * f + half) ^ sw) << 4;
      const u32x4 a = *reinterpret_cast<const u32x4*>(p + ch);
      const u32x4 b = *reinterpret_cast<const u32x4*>(q + ch);
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                  __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
  }

  // P (dS) as the second operand of `cols`. bf16 rounds it: the products take
  // bf16 operands and sum in fp32. A result is then off by 0.0021 to 0.0024 of its
  // norm, where its own rounding to bf16 is 0.0017; both parts of a split P would
  // take a second product each (one of the forward's two, three of the
  // passes' seven). fp32 keeps it.
  struct Probs {
    float x[BF ? 1 : 16];
    u32x4 b[BF ? 2 : 1];
  };
  __device__ static __forceinline__ void pack(Probs& p, const floatx16& s) {
    if constexpr (BF) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
        p.b[k] = u32x4{pack_bf16(s[8 * k], s[8 * k + 1]), pack_bf16(s[8 * k + 2], s[8 * k + 3]),
                       pack_bf16(s[8 * k + 4], s[8 * k + 5]), pack_bf16(s[8 * k + 6], s[8 * k + 7])};
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) p.x[r] = s[r];
    }
  }

  // 32 rows of an image, transposed, as the first operand of a `cols` product
  // (fp32 reads its elements in the product).
  struct ColFrag {
    u32x4 f[BF ? 2 * ND : 1];
    const char* at;
  };
  __device__ static __forceinline__ void load_cols(ColFrag& a, const char* img, int row0,
                                                   int lane) {
    if constexpr (BF) {
      // lane l of a 16-lane group supplies 4 elements of row l / 4, columns
      // 4 (l % 4); it receives column l of the 4 rows
      const int s = lane & 15, k = 4 * (lane >> 5) + (s >> 2);
      const int ch = 2 * ((lane >> 4) & 1) + ((s >> 1) & 1);
      const char* q = img + (row0 + k) * ROWB + (s & 1) * 8;
      const int sw = swz(k), sw8 = swz(k + 8);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const char* a0 = q + st * 16 * ROWB + (((4 * d + ch) ^ sw) << 4);
          const char* a1 = q + (st * 16 + 8) * ROWB + (((4 * d + ch) ^ sw8) << 4);
          const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)a0);
          const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)a1);
          typedef short short8_t __attribute__((ext_vector_type(8)));
          const short8_t v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          a.f[st * ND + d] = __builtin_bit_cast(u32x4, v);
        }
    } else {
      a.at = img + row0 * ROWB;
    }
  }
  // C[d] += A^T P
  __device__ static __forceinline__ void cols(floatx16 (&c)[ND], const ColFrag& a, const Probs& p,
                                              int lane) {
    if constexpr (BF) {
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int d = 0; d < ND; ++d)
          c[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              __builtin_bit_cast(bf16x8, a.f[st * ND + d]), __builtin_bit_cast(bf16x8, p.b[st]),
              c[d], 0, 0, 0);
    } else {
      const int half = lane >> 5, col = lane & 31;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int k = 8 * (r >> 2) + 4 * half + (r & 3);
        const char* q = a.at + k * ROWB + (col & 3) * 4;
        const int sw = swz(k);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const float x = *reinterpret_cast<const float*>(q + (((8 * d + (col >> 2)) ^ sw) << 4));
          c[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p.x[r], c[d], 0, 0, 0);
        }
      }
    }
  }

  // Stores a transposed result (lane: column l % 32 = one output row, rows
  // = its elements) times f to `row`, and what its rounding took off to `rest`
  // if that is given. bf16: the halves exchange 4-element groups first, so a
  // lane stores 16 bytes.
  __device__ static __forceinline__ void store_row(char* row, const floatx16 (&c)[ND], float f,
                                                   bool valid, int half, char* rest = nullptr) {
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      if constexpr (BF) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = c[d][8 * k + e] * f;
          const int at = (32 * d + 16 * k + 8 * half) * 2;
          store8(row + at, x, valid);
          if (rest != nullptr) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = rounding_rest(x[e]);
            store8(rest + at, x, valid);
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (valid)
            *reinterpret_cast<floatx4*>(row + (32 * d + 8 * k + 4 * half) * 4) =
                floatx4{c[d][4 * k] * f, c[d][4 * k + 1] * f, c[d][4 * k + 2] * f,
                        c[d][4 * k + 3] * f};
      }
    }
  }
  // The same in fp32, unscaled: a part's sums.
  __device__ static __forceinline__ void store_sums(float* row, const floatx16 (&c)[ND], bool valid,
                                                    int half) {
    if (!valid) return;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<floatx4*>(row + 32 * d + 8 * k + 4 * half) =
            floatx4{c[d][4 * k], c[d][4 * k + 1], c[d][4 * k + 2], c[d][4 * k + 3]};
  }
  // 8 elements of a row from both halves' groups of 4
  __device__ static __forceinline__ void store8(char* p, const float (&x)[8], bool valid) {
    const u32x2 a = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    const u32x2 b = {pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const auto y = __builtin_amdgcn_permlane32_swap(a[e], b[e], false, false);
      o[e] = y[0];
      o[2 + e] = y[1];
    }
    if (valid) *reinterpret_cast<u32x4*>(p) = o;
  }
};

// ---- relative position bias ------------------------------------------------
// The bias of a pair depends on t = key - query position alone, and is
// constant for t <= lo and for t >= hi. A workgroup spreads its head's column of
// the table over t once (times log2 e, as the scores enter exp2), 32 x 32
// blocks inside a constant side add one value, the others read LDS.
// (Reading the table through a bucket index costs a second LDS access an
// element.)
constexpr int BIAS_PAD = CROSS_BIAS_PAD;

__device__ __forceinline__ int bias_bucket(const CrossBias& b, int t) {
  int n, base = 0;
  if (b.bidirectional) {
    n = t < 0 ? -t : t;
    base = t > 0 ? b.side : 0;
  } else {
    n = t < 0 ? -t : 0;
  }
  if (n < b.exact) return base + n;
  int k = b.exact;
  const int f = b.side - b.exact;
#pragma unroll 8
  for (int i = 1; i < f; ++i) k += n >= b.border[i] ? 1 : 0;
  return base + k;
}

// entries of the spread table
__device__ __forceinline__ int bias_span(const CrossBias& b) { return b.hi - b.lo + 1 + 2 * BIAS_PAD; }

// a table entry as it enters exp2; entries below -1e30 mask
__device__ __forceinline__ float bias_entry(float x) {
  return x < -1e30f ? NEG_INF : x * LOG2E;
}

// Whether a constant side's entry may enter the exponent apart from the scores.
// A score is the fp32 sum of product and entry; next to an entry of -1e9 that sum
// has no bits of an ordinary product left, kept apart it has all: weights would
// differ from those of the same sums near the diagonal, and 2^(s - m) could pass
// 1 without bound. Up to 2^10 the two ways differ by less than 2^-13. (An entry of
// -INF masks: no sum to form.)
__device__ __forceinline__ bool side_apart(float entry) {
  return !(fabsf(entry) > 1024.f) || entry == NEG_INF;
}

// The entries of a head's constant sides, from its spread table, in scalar registers.
struct BiasSides {
  uint32_t lo = 0, hi = 0;
  uint32_t lo_apart = 0, hi_apart = 0;

  __device__ __forceinline__ static float read(const float* p) {
    return __uint_as_float(uni(__float_as_uint(*p)));
  }
  __device__ __forceinline__ void load(const float* tab, const CrossBias& b) {
    const float x = read(tab), y = read(tab + bias_span(b) - 1);
    lo = __float_as_uint(x);
    hi = __float_as_uint(y);
    lo_apart = uni(side_apart(x));
    hi_apart = uni(side_apart(y));
  }
  // The constant side that all t of [first, last] lie in, if it is taken apart:
  // -1, 1; else 0.
  __device__ __forceinline__ int of(const CrossBias& b, int first, int last) const {
    return lo_apart && last <= b.lo ? -1 : (hi_apart && first >= b.hi ? 1 : 0);
  }
  __device__ __forceinline__ float entry(int side) const {
    return __uint_as_float(side < 0 ? lo : hi);
  }
};

// the spread table of one head: tab[t - lo + BIAS_PAD]
__device__ __forceinline__ void bias_spread(float* tab, const CrossBias& b, int head, int heads,
                                            int tid, int nthreads) {
  const int n = bias_span(b);
  for (int i = tid; i < n; i += nthreads)
    tab[i] = bias_entry(b.table[int64_t(bias_bucket(b, i + b.lo - BIAS_PAD)) * heads + head]);
}

// x of the lane n to the right (left) in its row of 16 lanes, 0 past the end.
template <int N>
__device__ __forceinline__ float row_left(float x) {
  if constexpr (N == 0) return x;
  else return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
      0, __builtin_bit_cast(int, x), 0x100 + N, 0xf, 0xf, true));
}
template <int N>
__device__ __forceinline__ float row_right(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
      0, __builtin_bit_cast(int, x), 0x110 + N, 0xf, 0xf, true));
}

// Sums of a 32 x 32 block (lane: column l % 32, register r: row 8 (r / 4) +
// 4 half + r % 4) along its diagonals: lane u gets the sum of all elements with
// column - row = u - 32. A row is shifted onto the first one inside each 16
// lanes, what falls off goes to the next 16 diagonals down; then the halves (4
// rows apart) and the 16-column groups are joined. About 50 vector
// instructions; adding each element to its sum in LDS took 16 LDS atomics of
// some 250 cycles.
template <int R>
__device__ __forceinline__ void diag_row(float (&x)[3], float s) {
  constexpr int M = R / 16, N = R % 16;
  x[M] += row_left<N>(s);
  if constexpr (N > 0) x[M + 1] += row_right<16 - N>(s);
}
__device__ __forceinline__ float diagonal_sums(const floatx16& s, int lane) {
  float x[3] = {0.f, 0.f, 0.f};
  diag_row<0>(x, s[0]);
  diag_row<1>(x, s[1]);
  diag_row<2>(x, s[2]);
  diag_row<3>(x, s[3]);
  diag_row<8>(x, s[4]);
  diag_row<9>(x, s[5]);
  diag_row<10>(x, s[6]);
  diag_row<11>(x, s[7]);
  diag_row<16>(x, s[8]);
  diag_row<17>(x, s[9]);
  diag_row<18>(x, s[10]);
  diag_row<19>(x, s[11]);
  diag_row<24>(x, s[12]);
  diag_row<25>(x, s[13]);
  diag_row<26>(x, s[14]);
  diag_row<27>(x, s[15]);
  // x[m] of half h and column group g: diagonal 16 g + lane % 16 - 16 m - 4 h
  float y[3], fall = 0.f;
#pragma unroll
  for (int m = 0; m < 3; ++m) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[m]), __float_as_uint(x[m]),
                                                    false, false);
    const float up = __uint_as_float(r[1]);
    y[m] = __uint_as_float(r[0]) + row_left<4>(up) + fall;
    fall = row_right<12>(up);
  }
  const int G = lane >> 4;
  float v = 0.f;
#pragma unroll
  for (int m = 0; m < 3; ++m) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(y[m]), __float_as_uint(y[m]),
                                                    false, false);
    v += G == 2 - m ? __uint_as_float(r[0]) : 0.f;
    v += G == 3 - m ? __uint_as_float(r[1]) : 0.f;
  }
  return v;
}

// Sums of dS by t for the bias gradient, an array of bias_span entries for each
// wave: every sum's order is fixed. What falls in a constant side is summed in
// registers.
template <int NW>
struct BiasSums {
  float* arrays;
  float* mine;
  int span;
  float lo, hi;

  __device__ __forceinline__ void init(float* at, const CrossBias& b, int wave) {
    arrays = at;
    span = bias_span(b);
    mine = at + wave * span;
    lo = hi = 0.f;
  }
  __device__ __forceinline__ void clear(int tid) {
    for (int x = tid; x < NW * span; x += 64 * NW) arrays[x] = 0.f;
    lo = hi = 0.f;
  }
  // Adds a block (lane: key, registers: queries) whose corner (first key, first
  // query) has t = tb, inside [lo - 32, hi + 32].
  __device__ __forceinline__ void add(const CrossBias& b, const floatx16& s, int tb, int lane) {
    const float v = diagonal_sums(s, lane);
    if (lane > 0) mine[tb - 32 + lane - b.lo + BIAS_PAD] += v;
  }
  // Joins the arrays by t and writes the sum of every bucket. Called by the whole
  // workgroup, whose arrays are then free (behind a barrier). A side's buckets are
  // runs of t.
  __device__ __forceinline__ void flush(const CrossBias& b, float* out, int tid, int lane,
                                        int wave) {
    lo = group_sum<64>(lo);
    hi = group_sum<64>(hi);
    __syncthreads();
    for (int x = tid; x < span; x += 64 * NW) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) v += arrays[w * span + x];
      arrays[x] = v;
    }
    __syncthreads();
    float* ends = arrays + span;  // [NW][2]
    if (lane == 0) {
      ends[2 * wave] = lo;
      ends[2 * wave + 1] = hi;
    }
    __syncthreads();
    const float* tab = arrays + BIAS_PAD - b.lo;  // by t
    float below = 0.f, above = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      below += ends[2 * w];
      above += ends[2 * w + 1];
    }
    // eight lanes a bucket
    for (int x = tid; x < 8 * b.buckets; x += 64 * NW) {
      // distances [n0, n1) of the bucket; the last one of a side is open
      const int k = x >> 3, j = x & 7;
      const int u = k % b.side;
      const bool ahead = k >= b.side, last = u == b.side - 1;
      const int n0 = u <= b.exact ? u : b.border[u - b.exact];
      const int n1 = last ? 0 : (u < b.exact ? u + 1 : b.border[u - b.exact + 1]);
      float v = 0.f;
      if (!ahead) {
        const int t0 = last ? b.lo - BIAS_PAD : 1 - n1;
        for (int t = t0 + j; t <= -n0; t += 8) v += tab[t];
        if (last && j == 0) v += below;
        if (!b.bidirectional && u == 0) {  // keys ahead share the bucket of t = 0
          for (int t = 1 + j; t <= b.hi + BIAS_PAD; t += 8) v += tab[t];
          if (j == 0) v += above;
        }
      } else {
        const int t1 = last ? b.hi + BIAS_PAD : n1 - 1;
        for (int t = max(n0, 1) + j; t <= t1; t += 8) v += tab[t];
        if (last && j == 0) v += above;
      }
      v = group_sum<8>(v);
      if (j == 0) out[k] = v;
    }
  }
};

}  // namespace
}  // namespace abft
