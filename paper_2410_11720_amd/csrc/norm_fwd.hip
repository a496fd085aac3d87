// Layer norm forward, alone or behind the sum of a residual and a dropped-out
// input:
//   h = round(residual + dropout(x)) (or x), y = (h - mean) / sqrt(var + eps) w + b
// A row is held in the registers of LPR lanes from its one reading to its one
// writing; mean and variance are two sums over them. Bound by memory (bf16, alone: 8192
// x 768 8.2 us, 3.1 TB/s; 4096 x 4096 15.3 us, 4.4 TB/s; with residual and dropout 4096 x
// 5120 35 us, 4.8 TB/s).
#include <algorithm>

#include "rows.hpp"

namespace abft {
namespace {

// A row as it is read.
template <typename T, typename S, int KIND, int MODE> struct FwdLine {
  Chunk<T> x[S::NV], res[KIND == NORM_ALONE ? 1 : S::NV];
  bool ok;

  __device__ __forceinline__ void read(const NormArgs& a, const Place<T, S>& p, int row) {
    const RowAt at = row_at(a.tokens, min(row, a.rows - 1));
    ok = row < a.rows && (!a.lens || int(at.t) < a.lens[at.b]);
    const Line<T, S, MODE> px(a.x, at, ok, a.cols), pr(a.res, at, ok, a.cols);
#pragma unroll
    for (int j = 0; j < S::NV; ++j) {
      px.load(x[j], p, j);
      if constexpr (KIND != NORM_ALONE) pr.load(res[j], p, j);
    }
  }
};

// A value that a wave's lanes share, in a scalar register.
template <typename S> __device__ __forceinline__ float scalar(float x) {
  if constexpr (S::LPR == 0 || S::LPR >= 64)
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
  return x;
}

// The row after the present one is read ahead.
// (rows of several waves in bf16, or alone: five waves a SIMD, as many as a CU is given,
// which 96 registers allow; 4096 x 5120 with residual and dropout 43 us with 104, 34 with
// 96; 4096 x 8191 alone in fp32 62.0 and 61.5)
template <typename T> constexpr int FIVE = sizeof(T) == 2 ? 5 : 4;
template <typename T, typename S, int KIND, int MODE>
__global__ __launch_bounds__(S::LPR ? 256 : 1024,
                             S::LPR ? 1 : (MODE == ROWS_CHUNKS ? FIVE<T> : KIND == NORM_ALONE ? 5 : 4))
void norm_fwd_kernel(NormArgs a, ShapeAt shape) {
#pragma clang fp contract(off)  // (the same bits from every form; fused where written so)
  constexpr int NV = S::NV;
  __shared__ float2 sh[2][16];
  const Place<T, S> p(shape.lanes, a.cols);
  const int waves = shape.lanes / 64;
  const int step = gridDim.x * shape.rows;
  int row = blockIdx.x * shape.rows + p.slot, turn = 0;
  FwdLine<T, S, KIND, MODE> cur, next;
  cur.read(a, p, row);
  uint64_t seed = 0, offset = 0;
  if constexpr (KIND == NORM_DROPOUT) {
    seed = a.drop.rng[0];
    offset = a.drop.rng[1];
  }
  float w[NV][8], bias[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = p.col(j);
    load_params(w[j], a.weight, a.weight_bf16, col, a.cols - col, 1.f);
    load_params(bias[j], a.bias, a.weight_bf16, col, a.cols - col, 0.f);
  }
  const float inv_n = 1.f / float(a.cols);
  // (the workgroup's waves take as many turns: they meet in the sums)
  for (int first = blockIdx.x * shape.rows; first < a.rows; first += step, row += step, cur = next) {
    next.read(a, p, row + step);
    const RowAt at = row_at(a.tokens, min(row, a.rows - 1));
    const Line<T, S, MODE> py(a.y, at, row < a.rows, a.cols);
    const Line<T, S, MODE> ph(a.h, at, row < a.rows, a.cols);
    float v[NV][8];
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      settle<MODE>(cur.x[j], p, j, cur.ok);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = cur.x[j].get(e);
      if constexpr (KIND != NORM_ALONE) {
        if constexpr (KIND == NORM_DROPOUT)
          drop(v[j], a.drop, seed, offset, row, p.lane + j * p.lanes);
        settle<MODE>(cur.res[j], p, j, cur.ok);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = cur.res[j].get(e) + v[j][e];
        // the norm is that of the sum as it is stored, the one the backward and the
        // next layer read
        Chunk<T> c;
        c.set(v[j]);
        ph.store(c, p, j);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = c.get(e);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s.x += v[j][e];
    }
    // Mean and variance. The first mean's rounding is taken off both by the sum of the
    // differences. Where its square is above what that leaves of the variance, too few
    // bits are left: the row is taken less the corrected mean (a difference without
    // rounding, as its elements are then close to it; 0 throughout for a row of one value)
    // and summed again, once. Where the squares pass fp32's range the row is scaled by
    // 2^-80 and summed again.
    float mean, var, scale = 1.f, base = 0.f, by = 0.f;
    while (true) {
      mean = line_sum<S>(s, sh, waves, p.slot, turn).x * inv_n;
      s = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float2 t = make_float2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float d = v[j][e] - mean;
          if (MODE != ROWS_CHUNKS && p.col(j) + e >= a.cols) d = 0.f;
          t.x += d;
          t.y = fmaf(d, d, t.y);
        }
        s.x += p.has(j) ? t.x : 0.f;
        s.y += p.has(j) ? t.y : 0.f;
      }
      s = line_sum<S>(s, sh, waves, p.slot, turn);
      const float more = s.x * inv_n;
      var = fmaxf(fmaf(-more, more, s.y * inv_n), 0.f);
      float less = 0.f;
      if (is_finite(s.y) || scale != 1.f) {
        mean += more;
        if (is_nan(s.y)) var = s.y;  // (fmaxf takes the number)
        if (by == 1.f || !(more * more > var + (scale == 1.f ? a.eps : a.eps_scaled))) break;
        base = less = scalar<S>(mean);
        by = 1.f;
      } else {
        by = 0x1p-80f;
      }
      scale *= by;
      s = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float d = v[j][e] - less;
          if (MODE != ROWS_CHUNKS && p.col(j) + e >= a.cols) d = 0.f;
          v[j][e] = p.has(j) ? d * by : 0.f;
          s.x += v[j][e];
        }
    }
    // (a scaled row of variance 0 is one value throughout)
    const bool one = scale != 1.f && var == 0.f;
    const float r = 1.f / sqrtf(var + (scale == 1.f || one ? a.eps : a.eps_scaled));
    const float unscaled = (base + mean) * (scale == 1.f ? 1.f : 0x1p80f);
    const float2 st = cur.ok ? make_float2(unscaled, one ? r : r * scale) : make_float2(0.f, 0.f);
    if constexpr (MODE != ROWS_ANY)
      __builtin_amdgcn_raw_buffer_store_b64(
          __builtin_bit_cast(u32x2, st), bytes_at(a.stats, a.stats ? a.rows * 8u : 0u),
          p.lane == 0 && row < a.rows ? row * 8u : OUTSIDE, 0, 0);
    else if (a.stats && p.lane == 0 && row < a.rows)
      a.stats[row] = st;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf((v[j][e] - mean) * r, w[j][e], bias[j][e]);
      Chunk<T> c;
      c.set(o);
      c.keep(cur.ok);
      py.store(c, p, j);
    }
  }
}

// f(shape, its lanes and rows) for rows of whole chunks.
template <typename F> auto with_lines(int chunks, F f) {
  if (chunks <= 8) return f(Shape<8, 1>(), ShapeAt{8, 32});
  if (chunks <= 16) return f(Shape<16, 1>(), ShapeAt{16, 16});
  if (chunks <= 32) return f(Shape<32, 1>(), ShapeAt{32, 8});
  if (chunks <= 64) return f(Shape<32, 2>(), ShapeAt{32, 8});
  if (chunks <= 96) return f(Shape<32, 3>(), ShapeAt{32, 8});
  if (chunks <= 128) return f(Shape<64, 2>(), ShapeAt{64, 4});
  const int waves = (chunks + 127) / 128;
  return f(Shape<0, 2>(), ShapeAt{64 * waves, 1});
}

template <typename T, int KIND> hipError_t launch(const NormArgs& a, hipStream_t s) {
  return with_lines((a.cols + 7) / 8, [&](auto shape, ShapeAt at) {
    using S = decltype(shape);
    const int64_t wgs = (int64_t(a.rows) + at.rows - 1) / at.rows;
    // Waves of a CU, by what a lane holds, in whole workgroups: every CU has the same
    // number. Calls one after another in bf16: three chunks, 8192 x 768 with 8 waves 7.3,
    // 16 7.5 us, with dropout 12.7 and 13.6 (32768 rows 17.9 and 16.8); two, 8192 x 11072
    // with 20 waves 73.7, 16 82.1, 8 82.1 us, 4096 x 4096 14.8, 15.0, 17.0 (8192 x 2048
    // 15.6, 14.5, 16.9); 11 waves a row as 512 workgroups 73.7, as 465 75.0.
    constexpr int WAVES[] = {32, 20, 8};
    const int waves = at.threads() / 64, each = std::max(1, (WAVES[S::NV - 1] + waves / 2) / waves);
    const dim3 grid(int(std::min<int64_t>(wgs, 256 * each)));
    return start(a.mode == ROWS_CHUNKS  ? norm_fwd_kernel<T, S, KIND, ROWS_CHUNKS>
                 : a.mode == ROWS_WORDS ? norm_fwd_kernel<T, S, KIND, ROWS_WORDS>
                                        : norm_fwd_kernel<T, S, KIND, ROWS_ANY>,
                 grid, at.threads(), 0, s, a, at);
  });
}

template <typename T> hipError_t launch(const NormArgs& a, NormKind kind, hipStream_t s) {
  if (kind == NORM_ALONE) return launch<T, NORM_ALONE>(a, s);
  if (kind == NORM_RESIDUAL) return launch<T, NORM_RESIDUAL>(a, s);
  return launch<T, NORM_DROPOUT>(a, s);
}

}  // namespace

hipError_t launch_norm_fwd(const NormArgs& a, int dtype, NormKind kind, hipStream_t s) {
  return dtype == ABFT_BF16 ? launch<bf16_t>(a, kind, s) : launch<float>(a, kind, s);
}

}  // namespace abft
