// Layer norm backward: with xh = (h - mean) r and g = dy w of a row,
//   dh' = r (g - mean(g) - xh mean(g xh)) (+ dh, what comes from the sum itself),
//   dresidual = dh', dx = dropout(dh'); dweight = sum of dy xh, dbias = sum of dy
// over rows. A workgroup takes rows in turn, holds its columns' sums over them in
// registers and leaves them in the workspace; a second launch joins the
// workgroups' sums in one order (no atomics: results do not depend on
// scheduling). Bound by memory (bf16, alone: 8192 x 768 10.2 us, 3.7 TB/s; 4096 x 4096
// 21.1 us, 4.8 TB/s; with residual and dropout 4096 x 5120 44.8 us, 4.7 TB/s; the join 3 to
// 7.5 us).
#include <algorithm>

#include "rows.hpp"

namespace abft {
namespace {

// A row as it is read.
template <typename T, typename S, int KIND, int MODE> struct BwdLine {
  Chunk<T> dy[S::NV], h[S::NV], dh[KIND == NORM_ALONE ? 1 : S::NV];
  float2 st;
  bool ok;

  __device__ __forceinline__ void read(const NormArgs& a, const Place<T, S>& p, int row) {
    const int in = min(row, a.rows - 1);
    const RowAt at = row_at(a.tokens, in);
    ok = row < a.rows && (!a.lens || int(at.t) < a.lens[at.b]);
    const Line<T, S, MODE> pg(a.dy, at, ok, a.cols), ph(a.h, at, ok, a.cols), pd(a.dh, at, ok, a.cols);
    st = a.stats[in];
    // (a row that is not read has 0 in dy, dh and h; its statistics may be any row's)
    st.x = ok ? st.x : 0.f;
    st.y = ok ? st.y : 0.f;
#pragma unroll
    for (int j = 0; j < S::NV; ++j) {
      pg.load(dy[j], p, j);
      ph.load(h[j], p, j);
      if constexpr (KIND != NORM_ALONE) pd.load(dh[j], p, j);
    }
  }
};

// The row after the present one is read ahead. Rows above 8192 columns take up to 1024
// lanes of two chunks, 128 registers each: there g and xh are formed twice from what
// was read, and only bf16 rows without a residual are read ahead (4096 x 16384, with
// spills before: bf16 with residual and dropout 253 -> 145, fp32 alone 243 -> 164 us).
template <typename T, typename S, int KIND, int MODE>
__global__ __launch_bounds__(S::LPR ? 512 : 1024) void norm_bwd_kernel(NormArgs a, ShapeAt shape) {
#pragma clang fp contract(off)  // (the same bits from every form; fused where written so)
  constexpr int NV = S::NV;
  constexpr bool WIDE = S::LPR == 0 && NV > 1, AHEAD = !WIDE || (sizeof(T) == 2 && KIND == NORM_ALONE);
  __shared__ float2 sh[2][16];
  extern __shared__ float4 sums[];   // [rows][lanes NV][2] where there are several rows
  const Place<T, S> p(shape.lanes, a.cols);
  const int waves = shape.lanes / 64;
  const int step = gridDim.x * shape.rows;
  int row = blockIdx.x * shape.rows + p.slot, turn = 0;
  BwdLine<T, S, KIND, MODE> cur, next;
  if (AHEAD && a.rows > 0) cur.read(a, p, row);
  uint64_t seed = 0, offset = 0;
  if constexpr (KIND == NORM_DROPOUT) {
    seed = a.drop.rng[0];
    offset = a.drop.rng[1];
  }
  float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = p.col(j);
    load_params(w[j], a.weight, a.weight_bf16, col, a.cols - col, 1.f);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[j][e] = db[j][e] = 0.f;
  }
  const float inv_n = 1.f / float(a.cols);
  // (the workgroup's waves take as many turns: they meet in the sums)
  for (int first = blockIdx.x * shape.rows; first < a.rows; first += step, row += step) {
    if constexpr (AHEAD)
      next.read(a, p, row + step);
    else
      cur.read(a, p, row);
    const RowAt at = row_at(a.tokens, min(row, a.rows - 1));
    const Line<T, S, MODE> px(a.dx, at, row < a.rows, a.cols);
    const Line<T, S, MODE> pr(a.dres, at, row < a.rows, a.cols);
    const float mean = cur.st.x, r = cur.st.y;
    float g[WIDE ? 1 : NV][8], xh[WIDE ? 1 : NV][8];
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      settle<MODE>(cur.dy[j], p, j, cur.ok);
      settle<MODE>(cur.h[j], p, j, cur.ok);
      // (what is not in the row is 0 in dy, and must not be INF in xh)
      const float from = p.has(j) ? mean : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = cur.dy[j].get(e), gw = d * w[j][e];
        float x = (cur.h[j].get(e) - from) * r;
        if (MODE != ROWS_CHUNKS && p.col(j) + e >= a.cols) x = 0.f;
        dw[j][e] = fmaf(d, x, dw[j][e]);
        db[j][e] += d;
        s.x += gw;
        s.y = fmaf(gw, x, s.y);
        if constexpr (!WIDE) {
          xh[j][e] = x;
          g[j][e] = gw;
        }
      }
    }
    s = line_sum<S>(s, sh, waves, p.slot, turn);
    const float c1 = s.x * inv_n, c2 = s.y * inv_n;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (WIDE) {
        cur.dy[j].anew();
        cur.h[j].anew();
      }
      if constexpr (KIND != NORM_ALONE) settle<MODE>(cur.dh[j], p, j, cur.ok && a.dh.p);
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = WIDE ? (cur.h[j].get(e) - mean) * r : xh[j][e];
        const float gw = WIDE ? cur.dy[j].get(e) * w[j][e] : g[j][e];
        o[e] = r * fmaf(-x, c2, gw - c1);
        if constexpr (KIND != NORM_ALONE) o[e] += cur.dh[j].get(e);
      }
      // (a row that is not read has 0 in g only if the gain is finite: it is cleared)
      Chunk<T> c;
      c.set(o);
      if (!cur.ok) c.clear();
      if constexpr (KIND != NORM_ALONE) pr.store(c, p, j);
      if constexpr (KIND == NORM_DROPOUT) {
        // (in fp32 of what is stored: 4 bytes less of scratch in the widest form)
        if constexpr (sizeof(T) == 4)
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = c.get(e);
        drop(o, a.drop, seed, offset, row, p.lane + j * p.lanes);
        c.set(o);
        if (sizeof(T) == 2 && !cur.ok) c.clear();
      }
      px.store(c, p, j);
    }
    if constexpr (AHEAD) cur = next;
  }
  if (!a.dweight && !a.dbias) return;
  // the workgroup's sums: over its rows at a time, in their order
  float* out = a.part + int64_t(blockIdx.x) * a.stride;
  const int padded = norm_padded(a.cols);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float(&v)[NV][8] = k ? db : dw;
    if (shape.rows == 1) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (p.has(j)) {
          float4* to = reinterpret_cast<float4*>(out + k * padded) + 2 * (p.lane + j * p.lanes);
          to[0] = make_float4(v[j][0], v[j][1], v[j][2], v[j][3]);
          to[1] = make_float4(v[j][4], v[j][5], v[j][6], v[j][7]);
        }
      continue;
    }
    if (k) __syncthreads();
    const int width = p.lanes * NV * 2;   // (of four columns)
    float4* my = sums + p.slot * width;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      my[2 * (p.lane + j * p.lanes)] = make_float4(v[j][0], v[j][1], v[j][2], v[j][3]);
      my[2 * (p.lane + j * p.lanes) + 1] = make_float4(v[j][4], v[j][5], v[j][6], v[j][7]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < padded / 4; c += blockDim.x) {
      float4 t = sums[c];
      for (int q = 1; q < shape.rows; ++q) {
        const float4 x = sums[q * width + c];
        t = make_float4(t.x + x.x, t.y + x.y, t.z + x.z, t.w + x.w);
      }
      reinterpret_cast<float4*>(out + k * padded)[c] = t;
    }
  }
}

// Workgroups of the backward: each leaves sums of its own, so no more than one a CU, or
// two small ones.
constexpr int MOST_WGS = 256, MOST_SMALL_WGS = 512;

// dweight and dbias from the workgroups' sums: 32 columns a workgroup, 8 lanes of four
// columns each, the sums split over 128 such groups: at most 4 loads each, all in flight
// at once, then joined in LDS in their order.
constexpr int JOIN_NT = 1024, JOIN_COLS = 32, JOIN_GROUPS = JOIN_NT * 4 / JOIN_COLS;
static_assert(MOST_SMALL_WGS <= 4 * JOIN_GROUPS, "loads of a joining group");

__global__ __launch_bounds__(JOIN_NT) void norm_join_kernel(NormArgs a, int wgs) {
  __shared__ float sh[JOIN_GROUPS][JOIN_COLS], sh2[16][JOIN_COLS];
  const int c4 = threadIdx.x % 8, group = threadIdx.x / 8;
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  const float* at = a.part + blockIdx.x * JOIN_COLS + c4 * 4;
#pragma unroll 4
  for (int k = group; k < wgs; k += JOIN_GROUPS) {
    const float4 v = *reinterpret_cast<const float4*>(at + int64_t(k) * a.stride);
    t = make_float4(t.x + v.x, t.y + v.y, t.z + v.z, t.w + v.w);
  }
  *reinterpret_cast<float4*>(&sh[group][c4 * 4]) = t;
  __syncthreads();
  const int c = threadIdx.x % JOIN_COLS, q = threadIdx.x / JOIN_COLS;
  if (q < 16) {
    float v = sh[8 * q][c];
#pragma unroll
    for (int k = 1; k < 8; ++k) v += sh[8 * q + k][c];
    sh2[q][c] = v;
  }
  __syncthreads();
  if (q > 0) return;
  float v = sh2[0][c];
#pragma unroll
  for (int k = 1; k < 16; ++k) v += sh2[k][c];
  const int f = blockIdx.x * JOIN_COLS + c;
  const int padded = norm_padded(a.cols);
  float* to = f < padded ? a.dweight : a.dbias;
  const int col = f < padded ? f : f - padded;
  if (to && col < a.cols) to[col] = v;
}

// f(shape, its lanes and rows). Few chunks a lane: it holds their sums, 16 registers a
// chunk. As many rows a workgroup as fill it: its sums are written once for all of them
// (calls one after another, with the join: 4096 x 4096, 512 lanes a row, two rows a
// workgroup 23.9, one 24.7 us; 8192 x 768, a wave a row, eight rows 12.8, one 19.1), but
// no more than leave every CU a workgroup.
template <typename F> auto with_lines(int chunks, int64_t rows, F f) {
  auto at = [&](int lanes, int threads) {
    const int least = std::max(1, 64 / lanes), most = threads / lanes;
    const int64_t share = ((rows + 255) / 256 + least - 1) / least * least;
    return ShapeAt{lanes, int(std::max<int64_t>(least, std::min<int64_t>(most, share)))};
  };
  if (chunks <= 8) return f(Shape<8, 1>(), at(8, 256));
  if (chunks <= 16) return f(Shape<16, 1>(), at(16, 512));
  if (chunks <= 32) return f(Shape<16, 2>(), at(16, 512));
  if (chunks <= 64) return f(Shape<32, 2>(), at(32, 512));
  if (chunks <= 128) return f(Shape<64, 2>(), at(64, 512));
  if (chunks <= 1024) return f(Shape<0, 1>(), at((chunks + 63) / 64 * 64, 1024));
  return f(Shape<0, 2>(), at((chunks + 127) / 128 * 64, 1024));
}

int wgs_of(ShapeAt at, int64_t rows) {
  const int64_t most = at.threads() <= 256 ? MOST_SMALL_WGS : MOST_WGS;
  return int(std::max<int64_t>(1, std::min<int64_t>(most, (rows + at.rows - 1) / at.rows)));
}

template <typename T, int KIND> hipError_t launch(const NormArgs& a, hipStream_t s) {
  return with_lines((a.cols + 7) / 8, a.rows, [&](auto shape, ShapeAt at) {
    using S = decltype(shape);
    const int grid = wgs_of(at, a.rows);
    const size_t lds = at.rows > 1 ? size_t(at.threads()) * S::NV * 32 : 0;
    const hipError_t e =
        start(a.mode == ROWS_CHUNKS  ? norm_bwd_kernel<T, S, KIND, ROWS_CHUNKS>
              : a.mode == ROWS_WORDS ? norm_bwd_kernel<T, S, KIND, ROWS_WORDS>
                                     : norm_bwd_kernel<T, S, KIND, ROWS_ANY>,
              dim3(grid), at.threads(), lds, s, a, at);
    if (e != hipSuccess || (!a.dweight && !a.dbias)) return e;
    return start(norm_join_kernel, dim3(a.stride / JOIN_COLS), JOIN_NT, 0, s, a, grid);
  });
}

template <typename T> hipError_t launch(const NormArgs& a, NormKind kind, hipStream_t s) {
  if (kind == NORM_ALONE) return launch<T, NORM_ALONE>(a, s);
  if (kind == NORM_RESIDUAL) return launch<T, NORM_RESIDUAL>(a, s);
  return launch<T, NORM_DROPOUT>(a, s);
}

}  // namespace

int norm_bwd_wgs(int64_t rows, int cols) {
  return with_lines((cols + 7) / 8, rows, [&](auto, ShapeAt at) { return wgs_of(at, rows); });
}

hipError_t launch_norm_bwd(const NormArgs& a, int dtype, NormKind kind, hipStream_t s) {
  return dtype == ABFT_BF16 ? launch<bf16_t>(a, kind, s) : launch<float>(a, kind, s);
}

}  // namespace abft
