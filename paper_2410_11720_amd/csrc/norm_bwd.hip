// Layer norm backward: with xh = (h - mean) r and g = dy w of a row,
//   dh' = r (g - mean(g) - xh mean(g xh)) (+ dh, what comes from the sum itself),
//   dresidual = dh', dx = dropout(dh'); dweight = sum of dy xh, dbias = sum of dy
// over rows. A workgroup takes rows in turn, holds its columns' sums over them in
// registers and leaves them in the workspace; a second launch joins the
// workgroups' sums in one order (no atomics: results do not depend on
// scheduling). Bound by memory.
#include <algorithm>

#include "rows.hpp"

namespace abft {
namespace {

constexpr int MAX_WGS = 512;

template <typename T, typename S, int KIND>
__global__ __launch_bounds__(S::NT) void norm_bwd_kernel(NormArgs a) {
#pragma clang fp contract(off)  // (the same bits from every form; fused where written so)
  constexpr int LPR = S::LPR, NV = S::NV, R = S::R;
  __shared__ float2 sh[LPR > 64 ? 2 * LPR / 64 : 1];
  __shared__ float4 sums[R > 1 ? S::NT * NV * 2 : 1];
  const int lane = threadIdx.x % LPR;
  int turn = 0;
  float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = 8 * (lane + j * LPR);
    load_params(w[j], a.weight, a.weight_bf16, col, a.cols - col, 1.f);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[j][e] = db[j][e] = 0.f;
  }
  uint64_t seed = 0, offset = 0;
  if constexpr (KIND == NORM_DROPOUT) {
    seed = a.drop.rng[0];
    offset = a.drop.rng[1];
  }
  const float inv_n = 1.f / float(a.cols);
  const int step = gridDim.x * R;
  for (int row = blockIdx.x * R + threadIdx.x / LPR; row < a.rows; row += step) {
    RowAt at;
    at.b = a.tokens.quotient(row);
    at.t = row - at.b * a.tokens.d;
    T* dx = a.dx.p ? row_of<T>(a.dx, at) : nullptr;
    T* dres = a.dres.p ? row_of<T>(a.dres, at) : nullptr;
    if (a.lens && int(at.t) >= a.lens[at.b]) {
      Chunk<T> zero;
      zero.clear();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int col = 8 * (lane + j * LPR);
        if (dx) store_chunk(zero, dx + col, a.cols - col);
        if (KIND != NORM_ALONE && dres) store_chunk(zero, dres + col, a.cols - col);
      }
      continue;
    }
    const float2 st = a.stats[row];
    float g[NV][8], xh[NV][8];
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = 8 * (lane + j * LPR), m = a.cols - col;
      Chunk<T> c, ch;
      load_chunk(c, row_of<T>(a.dy, at) + col, m);
      load_chunk(ch, row_of<T>(a.h, at) + col, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = c.get(e);
        xh[j][e] = (ch.get(e) - st.x) * st.y;
        g[j][e] = d * w[j][e];
        dw[j][e] = fmaf(d, xh[j][e], dw[j][e]);
        db[j][e] += d;
        s.x += g[j][e];
        s.y = fmaf(g[j][e], xh[j][e], s.y);
      }
    }
    s = row_sum<LPR>(s, sh, turn);
    const float c1 = s.x * inv_n, c2 = s.y * inv_n;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = 8 * (lane + j * LPR), m = a.cols - col;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = st.y * fmaf(-xh[j][e], c2, g[j][e] - c1);
      Chunk<T> c;
      if constexpr (KIND != NORM_ALONE) {
        if (a.dh.p) {
          load_chunk(c, row_of<T>(a.dh, at) + col, m);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] += c.get(e);
        }
        if (dres) {
          c.set(o);
          store_chunk(c, dres + col, m);
        }
        if constexpr (KIND == NORM_DROPOUT) drop(o, a.drop, seed, offset, row, lane + j * LPR);
      }
      if (dx) {
        c.set(o);
        store_chunk(c, dx + col, m);
      }
    }
  }
  if (!a.dweight && !a.dbias) return;
  // the workgroup's sums: over its R rows at a time, in their order
  float* out = a.part + int64_t(blockIdx.x) * a.stride;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float(&v)[NV][8] = k ? db : dw;
    if constexpr (R > 1) {
      if (k) __syncthreads();
      float4* my = sums + (threadIdx.x / LPR) * (LPR * NV * 2);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        my[2 * (lane + j * LPR)] = make_float4(v[j][0], v[j][1], v[j][2], v[j][3]);
        my[2 * (lane + j * LPR) + 1] = make_float4(v[j][4], v[j][5], v[j][6], v[j][7]);
      }
      __syncthreads();
      const float* f = reinterpret_cast<const float*>(sums);
      for (int c = threadIdx.x; c < a.cols; c += S::NT) {
        float t = f[c];
        for (int q = 1; q < R; ++q) t += f[q * (LPR * NV * 8) + c];
        out[k * a.cols + c] = t;
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = 8 * (lane + j * LPR) + e;
          if (c < a.cols) out[k * a.cols + c] = v[j][e];
        }
    }
  }
}

// dweight and dbias from the workgroups' sums: 64 columns a workgroup, 16 lanes of
// four columns, the sums split over 16 such groups.
__global__ __launch_bounds__(256) void norm_join_kernel(NormArgs a, int wgs) {
  __shared__ float4 sh[256];
  const int c4 = threadIdx.x % 16, k0 = threadIdx.x / 16;
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  const float* at = a.part + blockIdx.x * 64 + c4 * 4;
  for (int k = k0; k < wgs; k += 16) {
    const float4 v = *reinterpret_cast<const float4*>(at + int64_t(k) * a.stride);
    t.x += v.x;
    t.y += v.y;
    t.z += v.z;
    t.w += v.w;
  }
  sh[threadIdx.x] = t;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const int f = blockIdx.x * 64 + threadIdx.x;
  const float* s = reinterpret_cast<const float*>(sh) + threadIdx.x;
  float v = s[0];
  for (int k = 1; k < 16; ++k) v += s[64 * k];
  if (f < a.cols) {
    if (a.dweight) a.dweight[f] = v;
  } else if (f < 2 * a.cols) {
    if (a.dbias) a.dbias[f - a.cols] = v;
  }
}

template <typename S> int wgs_of(int64_t rows) {
  return int(std::max<int64_t>(1, std::min<int64_t>(MAX_WGS, (rows + S::R - 1) / S::R)));
}

template <typename T, int KIND> hipError_t launch(const NormArgs& a, hipStream_t s) {
  return with_shape((a.cols + 7) / 8, [&](auto shape) {
    using S = decltype(shape);
    const int grid = wgs_of<S>(a.rows);
    norm_bwd_kernel<T, S, KIND><<<dim3(grid), S::NT, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.dweight && !a.dbias)) return e;
    norm_join_kernel<<<dim3(a.stride / 64), 256, 0, s>>>(a, grid);
    return hipGetLastError();
  });
}

template <typename T> hipError_t launch(const NormArgs& a, NormKind kind, hipStream_t s) {
  if (kind == NORM_ALONE) return launch<T, NORM_ALONE>(a, s);
  if (kind == NORM_RESIDUAL) return launch<T, NORM_RESIDUAL>(a, s);
  return launch<T, NORM_DROPOUT>(a, s);
}

}  // namespace

int norm_bwd_wgs(int64_t rows, int cols) {
  return with_shape((cols + 7) / 8, [&](auto shape) { return wgs_of<decltype(shape)>(rows); });
}

hipError_t launch_norm_bwd(const NormArgs& a, int dtype, NormKind kind, hipStream_t s) {
  return dtype == ABFT_BF16 ? launch<bf16_t>(a, kind, s) : launch<float>(a, kind, s);
}

}  // namespace abft
