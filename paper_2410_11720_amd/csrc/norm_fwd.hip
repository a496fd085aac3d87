// Layer norm forward, alone or behind the sum of a residual and a dropped-out
// input:
//   h = round(residual + dropout(x)) (or x), y = (h - mean) / sqrt(var + eps) w + b
// A row is held in the registers of LPR lanes from its one reading to its one
// writing; mean and variance are two sums over them. Bound by memory.
#include "rows.hpp"

namespace abft {
namespace {

template <typename T, typename S, int KIND>
__global__ __launch_bounds__(S::NT) void norm_fwd_kernel(NormArgs a) {
#pragma clang fp contract(off)  // (the same bits from every form; fused where written so)
  constexpr int LPR = S::LPR, NV = S::NV;
  __shared__ float2 sh[LPR > 64 ? 2 * LPR / 64 : 1];
  const int lane = threadIdx.x % LPR;
  int turn = 0;
  float w[NV][8], bias[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = 8 * (lane + j * LPR);
    load_params(w[j], a.weight, a.weight_bf16, col, a.cols - col, 1.f);
    load_params(bias[j], a.bias, a.weight_bf16, col, a.cols - col, 0.f);
  }
  uint64_t seed = 0, offset = 0;
  if constexpr (KIND == NORM_DROPOUT) {
    seed = a.drop.rng[0];
    offset = a.drop.rng[1];
  }
  const float inv_n = 1.f / float(a.cols);
  const int step = gridDim.x * S::R;
  for (int row = blockIdx.x * S::R + threadIdx.x / LPR; row < a.rows; row += step) {
    RowAt at;
    at.b = a.tokens.quotient(row);
    at.t = row - at.b * a.tokens.d;
    T* y = row_of<T>(a.y, at);
    T* hp = a.h.p ? row_of<T>(a.h, at) : nullptr;
    if (a.lens && int(at.t) >= a.lens[at.b]) {
      Chunk<T> zero;
      zero.clear();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int col = 8 * (lane + j * LPR);
        store_chunk(zero, y + col, a.cols - col);
        if (KIND != NORM_ALONE && hp) store_chunk(zero, hp + col, a.cols - col);
      }
      if (a.stats && lane == 0) a.stats[row] = make_float2(0.f, 0.f);
      continue;
    }
    float v[NV][8];
    const T* x = row_of<T>(a.x, at);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = 8 * (lane + j * LPR), m = a.cols - col;
      Chunk<T> c;
      load_chunk(c, x + col, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = c.get(e);
      if constexpr (KIND != NORM_ALONE) {
        if constexpr (KIND == NORM_DROPOUT) drop(v[j], a.drop, seed, offset, row, lane + j * LPR);
        load_chunk(c, row_of<T>(a.res, at) + col, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = plain_add(c.get(e), v[j][e]);
        // the norm is that of the sum as it is stored, the one the backward and the
        // next layer read
        c.set(v[j]);
        if (hp) store_chunk(c, hp + col, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = c.get(e);
      }
    }
    // Mean and variance. The first mean's rounding is taken off both by the sum of
    // the differences (a row of one large value has variance 0). Where the squares
    // pass fp32's range the row is scaled by 2^-80 and summed again.
    float mean, var, scale = 1.f;
    while (true) {
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) s.x += v[j][e];
      s = row_sum<LPR>(s, sh, turn);
      mean = s.x * inv_n;
      s = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int m = a.cols - 8 * (lane + j * LPR);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = e < m ? v[j][e] - mean : 0.f;
          s.x += d;
          s.y = fmaf(d, d, s.y);
        }
      }
      s = row_sum<LPR>(s, sh, turn);
      const float more = s.x * inv_n;
      var = fmaxf(fmaf(-more, more, s.y * inv_n), 0.f);
      const bool again = !is_finite(s.y) && scale == 1.f;
      if (!again) {
        mean += more;
        if (is_nan(s.y)) var = s.y;  // (fmaxf takes the number)
        break;
      }
      scale = 0x1p-80f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] *= scale;
    }
    const float r = 1.f / sqrtf(scale == 1.f ? var + a.eps : var);
    if (a.stats && lane == 0) a.stats[row] = make_float2(mean / scale, r * scale);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = 8 * (lane + j * LPR);
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf((v[j][e] - mean) * r, w[j][e], bias[j][e]);
      Chunk<T> c;
      c.set(o);
      store_chunk(c, y + col, a.cols - col);
    }
  }
}

template <typename T, int KIND> hipError_t launch(const NormArgs& a, hipStream_t s) {
  return with_shape((a.cols + 7) / 8, [&](auto shape) {
    using S = decltype(shape);
    const int64_t wgs = (int64_t(a.rows) + S::R - 1) / S::R;
    const int grid = int(wgs < 2048 ? wgs : 2048);
    norm_fwd_kernel<T, S, KIND><<<dim3(grid), S::NT, 0, s>>>(a);
    return hipGetLastError();
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
