// Attention over keys of another length, backward, from the forward's lse.
//
//   P_ij = 2^(s_ij log2 e - lse_i),  D_i = dO_i . O_i,  dP_ij = dO_i . v_j,
//   dS_ij = P_ij (dP_ij - D_i),
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,
//   dv_j = sum_i P_ij dO_i,  dtable[t] = sum over pairs of bucket t of dS_ij,
// with dk_j and dv_j summed over the query heads that share a key head.
//
// lse is one fp32 number: beside scores of 1e6 the logarithm of a row's sum has
// few bits left in it, beside 1e9 none, and the row's P sum to anything up to
// its number of keys. Where an lse is that large the query pass first sums its
// row's P, and both passes divide by the sum.
//
// Two passes, each of which owns what it sums (no atomics on memory, so
// results do not depend on the order of workgroups): a workgroup of the query
// pass owns 32 to 128 queries and runs over the keys (dq; it leaves -lse and -D
// for the other pass), one of the key pass owns 32 to 128 keys and runs over the
// queries of all heads that share them (dk, dv, dtable). Small grids split the
// other axis too, over the waves of a workgroup and over workgroups (cross_plan).
// The price of two passes is a second S and dP (14 d flops a pair against 10 d in
// one). Matrix cores are busy for 41% and 49% of the passes' cycles at 4 x 2048
// queries over 1024 keys, 32 heads on 8, head dim 128, the vector ALU for 43% and
// 28%: 268 and 303 us (medians), 0.77 and 0.91 PFLOP/s of bf16. 8 x 1024 causal,
// 12 heads, head dim 64, with a bias: 44 and 61 us.
#include "cross_tile.hpp"

namespace abft {
namespace {

// Whether a product's fragments are read ahead of the work in front of it: where
// the registers last (head dim 64 in bf16; cross attention of 8 x 512 over 1000,
// 12 heads: 73 -> 68 us).
template <typename T, int D>
constexpr bool read_ahead() { return D * sizeof(T) == 128; }

// |lse| past which a row's P are summed: below, its rounding moves them by less than
// 2^-12 in bf16, an eighth of their own rounding, and 2^-16 in fp32. (The sums cost a wave a
// third pass over its keys: 8 x 512 over 1000, 12 heads, all rows large: 75 -> 119
// us, with a bias of -1e9 throughout 100 -> 336.)
template <typename T>
constexpr float large_lse() { return sizeof(T) == 2 ? 4096.f : 256.f; }
__device__ __forceinline__ float inverse(float total) { return total == 0.f ? 1.f : 1.f / total; }

// Sum of 2^(s - lse) over the lane's row i, for the 32 rows of a wave from w0 on:
// keys straight from memory, an entry of the bias from its bucket. Slow, and
// rare: the passes' own loops do without.
template <typename T, int D, bool BIAS>
__device__ __forceinline__ float row_total(const CrossArgs& a, const typename CrossTile<T, D>::RowFrag& q,
                                        float nl, int b, int h, int w0, int end, int lane) {
  using Tile = CrossTile<T, D>;
  const int half = lane >> 5, i = w0 + (lane & 31);
  const int len = seq_len(a, b), start = seq_start(a, b);
  const int limit = a.causal ? min(len, start + i + 1) : len;
  const char* kp = a.k.p + b * a.k.b + (h / a.group) * a.k.h;
  const float c = a.scale * LOG2E;
  auto entry = [&](int bucket) {
    return bias_entry(a.bias.table[int64_t(bucket) * a.nh + h]);
  };
  float total = 0.f;
  for (int k0 = 0; k0 < end; k0 += 32) {
    typename Tile::RowFrag kf;
    Tile::load_row(kf, kp + int64_t(min(k0 + (lane & 31), len - 1)) * a.k.t, half);
    floatx16 s = floatx16{};
    Tile::rows(s, kf, q);
    float ce = c, off = nl;
    if constexpr (BIAS) {
      const int tb = k0 - start - w0;
      float x = 0.f;
      bool apart = false;
      if (tb + 31 <= a.bias.lo || tb - 31 >= a.bias.hi) {
        x = entry(bias_bucket(a.bias, tb));
        apart = side_apart(x);
      }
      if (apart) {
        off += x;
      } else {
        ce = 1.f;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[r] = fmaf(s[r], c, entry(bias_bucket(a.bias, k0 + 8 * (r >> 2) + 4 * half + (r & 3) -
                                                             start - i)));
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const bool seen = k0 + 8 * (r >> 2) + 4 * half + (r & 3) < limit;
      total += seen ? exp2_hw(fmaf(s[r], ce, off)) : 0.f;
    }
  }
  return half_sum(total);
}

template <typename T>
__device__ __forceinline__ void store4(char* p, floatx4 v) {
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  else
    *reinterpret_cast<floatx4*>(p) = v;
}

// ---- query pass -----------------------------------------------------------
// WV: workgroups a CU that its registers allow; at three nothing is read ahead.
// (With a bias four forms spill: at three a CU 1 and 5 registers, at head dim 128
// where waves share queries 5 and 9.)
template <typename T, int D, bool BIAS, int NQ, int KS, int WV>
__global__ __launch_bounds__(64 * NQ * KS, WV) void
cross_bwd_q_kernel(CrossArgs a) {
  using Tile = CrossTile<T, D>;
  constexpr int NW = NQ * KS, KT = cross_rows(sizeof(T), KS), NB = KT / 32 / KS;
  constexpr int IMG = KT * Tile::ROWB;
  constexpr bool AHEAD = WV < 3 && read_ahead<T, D>();
  __shared__ float row_sum[KS > 1 ? NW * 64 : 1];
  extern __shared__ __align__(1024) char smem[];
  float* tab = reinterpret_cast<float*>(smem + 4 * IMG);

  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), half = lane >> 5;
  const int nbk = a.B * a.kvh, ntile = cross_tiles(a.Sq, 32 * NQ);
  const int bk = blockIdx.x % nbk, y = blockIdx.x / nbk;
  const int b = bk / a.kvh, kv = bk % a.kvh, h = kv * a.group + y % a.group;
  const int part = y / (a.group * ntile);
  int tile = y / a.group % ntile;
  if (a.causal) tile = ntile - 1 - tile;
  const int q0 = tile * 32 * NQ;
  const int len = seq_len(a, b), start = seq_start(a, b);
  int kend = len;
  if (a.causal) kend = min(kend, start + min(q0 + 32 * NQ, a.Sq));
  kend = max(kend, 0);
  const int nt = (kend + KT - 1) / KT;
  // the workgroup's tiles
  const int t0 = int(int64_t(nt) * part / a.q_parts), t1 = int(int64_t(nt) * (part + 1) / a.q_parts);
  const int qw = wave % NQ, ks = wave / NQ;
  const int w0 = q0 + 32 * qw, i = w0 + (lane & 31), ic = min(i, a.Sq - 1);
  const bool valid = i < a.Sq;
  int wend = len;
  if (a.causal) wend = min(wend, start + min(w0 + 32, a.Sq));
  if (w0 >= a.Sq) wend = 0;
  const int limit = a.causal ? min(len, start + i + 1) : len;

  const char* kp = a.k.p + b * a.k.b + kv * a.k.h;
  const char* vp = a.v.p + b * a.v.b + kv * a.v.h;
  const uint32_t lds0 = lds_addr(smem);
  auto issue = [&](int t) {
    const uint32_t to = lds0 + (t & 1) * 2 * IMG;
    Tile::template issue<KT, NW>(kp + int64_t(t) * KT * a.k.t, a.k.t, len - t * KT, to, wave, lane);
    Tile::template issue<KT, NW>(vp + int64_t(t) * KT * a.v.t, a.v.t, len - t * KT, to + IMG, wave,
                                lane);
  };
  if (t1 > t0) issue(t0);

  typename Tile::RowFrag q, g;
  Tile::load_row(q, a.q.p + b * a.q.b + h * a.q.h + int64_t(ic) * a.q.t, half);
  Tile::load_row(g, a.dout.p + b * a.dout.b + h * a.dout.h + int64_t(ic) * a.dout.t, half);
  float nl, nd;
  {
    typename Tile::RowFrag o;
    Tile::load_row(o, a.o.p + b * a.o.b + h * a.o.h + int64_t(ic) * a.o.t, half);
    nd = Tile::dot_row(g, o);
    if (sizeof(T) == 2 && a.rest != nullptr) {
      // dP - D cancels, so D is formed from O before its rounding
      Tile::load_row(o, a.rest + ((int64_t(b) * a.nh + h) * a.Sq + ic) * Tile::ROWB, half);
      nd += Tile::dot_row(g, o);
    }
    nd = -half_sum(nd);
    const float lse = a.lse[(int64_t(b) * a.nh + h) * a.Sq + ic];
    // rows without keys (whatever they hold) and rows past the last query: P = 0
    nl = valid && lse != NEG_INF ? -lse : NEG_INF;
    if (nl == NEG_INF) {
      nd = 0.f;
      Tile::zero_row(g);
    }
  }
  if constexpr (BIAS) bias_spread(tab, a.bias, h, a.nh, tid, 64 * NW);
  float sum = 0.f;   // of the row's dS
  float norm = 1.f;  // what its P (and with them dS) are to be multiplied by
  if (__any(nl != NEG_INF && !(fabsf(nl) <= large_lse<T>())))
    norm = inverse(row_total<T, D, BIAS>(a, q, nl, b, h, w0, wend, lane));

  // rows between the last query and the end of the key pass's tiles: P = 0
  if (part == 0 && q0 + 32 * NQ >= a.Sq)
    for (int x = q0 + 32 * NQ + tid; x < a.q_pad; x += 64 * NW) {
      const int64_t at = (int64_t(b) * a.nh + h) * a.q_pad + x;
      a.nlse[at] = NEG_INF;
      a.ndelta[at] = 0.f;
      a.norm[at] = 1.f;
    }
  const float nd0 = nd;
  // a row's sum over its KS waves (all call it together, behind the last use of
  // the sums before)
  auto join_sum = [&](float x) {
    x = half_sum(x);
    if constexpr (KS > 1) {
      row_sum[wave * 64 + lane] = x;
      __syncthreads();
      x = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) x += row_sum[(qw + k * NQ) * 64 + lane];
      __syncthreads();
    }
    return x;
  };

  // -D in every register of a block: what the products that form dP - D start
  // from (where registers last; else moves before each product, a quarter of the
  // vector instructions at head dim 64)
  floatx16 minus_d = nd;
  floatx16 dq[Tile::ND];
#pragma unroll
  for (int d = 0; d < Tile::ND; ++d) dq[d] = floatx16{};
  const float c = a.scale * LOG2E;
  for (int t = t0; t < t1; ++t) {
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < t1) issue(t + 1);
    const int k0 = t * KT + 32 * NB * ks;  // the wave's keys of the tile
    const char* img = smem + (t & 1) * 2 * IMG + 32 * NB * ks * Tile::ROWB;
    const bool masked = k0 + 32 * NB > len || (a.causal && k0 + 32 * NB - 1 > start + w0);
    // rows of few keys (one tile) sum their dS first and correct D by it: there
    // the rounding of single P shows in dq
    for (int sweep = (KS > 1 ? nt == 1 : wend <= KT) ? 0 : 1; sweep < 2; ++sweep) {
      asm volatile("" ::: "memory");  // (reads of the image stay in the loop: they need registers)
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        if (k0 >= wend) continue;
        floatx16 s = floatx16{}, dp;
        typename Tile::RowFrag kf, vf;
        Tile::load_rows(kf, img, 32 * n, lane);
        Tile::load_rows(vf, img + IMG, 32 * n, lane);
        float x = 0.f;
        int tb = 0;
        if constexpr (BIAS) {
          tb = k0 + 32 * n - start - w0;  // the block spans [tb - 31, tb + 31]
          x = tab[tb < a.bias.hi ? 0 : bias_span(a.bias) - 1];  // the side's entry, if in one
        }
        issue_loads<AHEAD>();
        Tile::rows(s, kf, q);
        if constexpr (AHEAD) {
          dp = minus_d;
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) dp[r] = nd;
        }
        Tile::rows(dp, vf, g);
        typename Tile::ColFrag kc;
        if constexpr (AHEAD) Tile::load_cols(kc, img, 32 * n, lane);
        issue_loads<AHEAD>();
        float ce = c, off = nl;
        if constexpr (BIAS) {
          if ((tb + 31 <= a.bias.lo || tb - 31 >= a.bias.hi) && uni(side_apart(x))) {
            off += x;
          } else {
            ce = 1.f;
            tb = clampi(tb, a.bias.lo - 32, a.bias.hi + 32);  // (where the table has entries)
            const float* p = tab + (tb - (lane & 31) + 4 * half - a.bias.lo + BIAS_PAD);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], c, p[8 * (r >> 2) + (r & 3)]);
          }
        }
        if (masked) {
          const int lim = limit - k0 - 32 * n - 4 * half;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < lim ? s[r] : NEG_INF;
        }
        for (int r = 0; r < 16; ++r) {
          s[r] = exp2_hw(fmaf(s[r], ce, off)) * dp[r];
          sum += s[r];
        }
        if (sweep == 0) continue;
        typename Tile::Probs p;
        Tile::pack(p, s);
        if constexpr (!AHEAD) Tile::load_cols(kc, img, 32 * n, lane);
        Tile::cols(dq, kc, p, lane);
      }
      if (sweep == 0) {
        nd -= join_sum(sum) * norm;
        sum = 0.f;
        minus_d = nd;
      }
    }
  }
  if constexpr (KS > 1) {
    float* box = reinterpret_cast<float*>(smem) + lane;
    constexpr int BOX = 64 * 16 * Tile::ND;
    static_assert(NQ * (KS - 1) * BOX * 4 <= 4 * IMG, "the tiles' space holds the boxes");
    sum = join_sum(sum);  // (a barrier: the tiles are no longer read)
    if (ks > 0) {
#pragma unroll
      for (int e = 0; e < 16 * Tile::ND; ++e)
        box[(wave - NQ) * BOX + 64 * e] = dq[e / 16][e % 16];
    }
    __syncthreads();
    if (ks > 0) return;
#pragma unroll
    for (int k = 1; k < KS; ++k)
#pragma unroll
      for (int e = 0; e < 16 * Tile::ND; ++e)
        dq[e / 16][e % 16] += box[(wave + (k - 1) * NQ) * BOX + 64 * e];
  } else {
    sum = half_sum(sum);
  }
  // For the key pass: -lse, what P is multiplied by, and D so that the row's dS sum
  // to zero as they must. (O was formed from P rounded to bf16, which moves D by
  // 2^-9 of its terms; a bias gradient, the sum of many dS of either sign, was off
  // by 0.1%.)
  const int64_t row = int64_t(b) * a.nh + h, at = row * a.q_pad + i;
  nd -= sum * norm;
  if (a.q_parts == 1) {
    Tile::store_row(a.dq.p + b * a.dq.b + h * a.dq.h + int64_t(i) * a.dq.t, dq, a.scale * norm,
                    valid, half);
  } else {
    const int64_t rows = int64_t(a.B) * a.nh;
    Tile::store_sums(a.part_dq + ((part * rows + row) * a.Sq + i) * D, dq, valid, half);
    if (half == 0) a.part_sum[part * rows * a.q_pad + at] = nd0 - nd;
    nd = nd0;  // (cross_join_q_kernel takes the parts' sums off)
  }
  if (half == 0 && part == 0) {
    a.nlse[at] = nl;
    a.ndelta[at] = nd;
    a.norm[at] = norm;
  }
}

// Joins the query pass's parts in their order: dq, and -D less the sums of dS.
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_join_q_kernel(CrossArgs a) {
  const int64_t x = int64_t(blockIdx.x) * 256 + threadIdx.x, rows = int64_t(a.B) * a.nh;
  const int64_t r = x / (D / 4);
  const int e = int(x % (D / 4)) * 4;
  if (r >= rows * a.Sq) return;
  const int64_t bh = r / a.Sq, i = r % a.Sq;
  floatx4 v = {};
  for (int p = 0; p < a.q_parts; ++p)
    v += *reinterpret_cast<const floatx4*>(a.part_dq + (p * rows * a.Sq + r) * D + e);
  const int b = int(bh / a.nh), h = int(bh % a.nh);
  store4<T>(a.dq.p + b * a.dq.b + h * a.dq.h + i * a.dq.t + e * int(sizeof(T)),
            v * (a.scale * a.norm[bh * a.q_pad + i]));
  if (e == 0) {
    float s = 0.f;
    for (int p = 0; p < a.q_parts; ++p) s += a.part_sum[(p * rows + bh) * a.q_pad + i];
    a.ndelta[bh * a.q_pad + i] -= s;
  }
}

// Sums the key pass's partial bias gradients of one head in a fixed order.
__device__ __forceinline__ void sum_dbias(const float* part, float* dbias, int n, int buckets,
                                          int heads, int h) {
  __shared__ float sh[256];
  const int lanes = 256 / buckets;  // partial sums of a bucket
  const int k = threadIdx.x % buckets, j = threadIdx.x / buckets;
  float v = 0.f;
  if (j < lanes) {
    const float* p = part + int64_t(h) * n * buckets + k;
    int x = j;
    for (; x + 7 * lanes < n; x += 8 * lanes) {  // eight loads at a time
      float y[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) y[u] = p[int64_t(x + u * lanes) * buckets];
#pragma unroll
      for (int u = 0; u < 8; ++u) v += y[u];
    }
    for (; x < n; x += lanes) v += p[int64_t(x) * buckets];
  }
  sh[threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.x < buckets) {
    for (int x = 1; x < lanes; ++x) v += sh[x * buckets + threadIdx.x];
    dbias[int64_t(threadIdx.x) * heads + h] = v;
  }
}

__global__ __launch_bounds__(256) void cross_dbias_kernel(const float* part, float* dbias, int n,
                                                          int buckets, int heads) {
  sum_dbias(part, dbias, n, buckets, heads, blockIdx.x);
}

// Joins the key pass's parts in their order: dk (y = 0) or dv (1), and the bias
// gradient of head x (2), from n partial sums.
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_join_kv_kernel(CrossArgs a, int n) {
  if (blockIdx.y == 2) {
    if (blockIdx.x < uint32_t(a.nh))
      sum_dbias(a.dbias_part, a.dbias, n, a.bias.buckets, a.nh, blockIdx.x);
    return;
  }
  const int64_t x = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t r = x / (D / 4), rows = int64_t(a.B) * a.kvh * a.Sk;
  const int e = int(x % (D / 4)) * 4;
  if (r >= rows) return;
  const float* from = blockIdx.y == 0 ? a.part_dk : a.part_dv;
  const CrossTensor& to = blockIdx.y == 0 ? a.dk : a.dv;
  floatx4 v = {};
  for (int p = 0; p < a.kv_parts; ++p)
    v += *reinterpret_cast<const floatx4*>(from + (p * rows + r) * D + e);
  const int64_t bh = r / a.Sk, j = r % a.Sk;
  const int b = int(bh / a.kvh), h = int(bh % a.kvh);
  store4<T>(to.p + b * to.b + h * to.h + j * to.t + e * int(sizeof(T)),
            v * (blockIdx.y == 0 ? a.scale : 1.f));
}

// ---- key pass ---------------------------------------------------------------
// S = Q K^T, so that a lane holds the scores of one key (its mask is a bound on
// the query) and P and dS are the second operands of dV^T = dO^T P and
// dK^T = Q^T dS from registers.
// A workgroup has KW x QH waves: 32 KW keys, and QH waves on the same 32 that
// take different rows of a query tile and join their sums at the end.
// At head dim 128 the accumulators of both gradients and the keys' and values' own
// fragments do not fit 256 registers beside the scores (36 spilled, and the pass of
// 4 x 2048 queries over 1024 keys, 32 heads on 8, took more than twice as long). In
// bf16 the values' are read from LDS, which leaves room for one workgroup a CU, of 8
// waves (of 4 waves a third slower). fp32 runs one wave per SIMD.
// The forms that grids fill the chip with keep to their registers, but for fp32
// with a bias at head dim 128 (4 spilled). Some for small grids do not: bf16 at
// head dim 128, 2 x 4 waves with a bias (53 spilled) and 2 x 2 without (10); fp32 at
// head dim 64 without a bias spills 18 to 33 in all three.
template <typename T, int D, bool BIAS, int KW, int QH>
__global__ __launch_bounds__(64 * KW * QH, (sizeof(T) * D == 512 ? 1 : 2)) void
cross_bwd_kv_kernel(CrossArgs a) {
  using Tile = CrossTile<T, D>;
  constexpr int QT = cross_rows(sizeof(T), QH), NB = QT / 32 / QH, NW = KW * QH, KEYS = 32 * KW;
  constexpr int IMG = QT * Tile::ROWB;
  constexpr int NS = cross_stats(QT);
  constexpr int STAGE = 2 * IMG + 12 * NS;  // Q, dO, -lse, -D and norm of a tile
  constexpr bool KLDS = cross_k_in_lds(sizeof(T), D, QH, BIAS);
  constexpr bool VLDS = cross_v_in_lds(sizeof(T), D), AHEAD = read_ahead<T, D>();
  extern __shared__ __align__(1024) char smem[];
  const char* vimg = smem + 2 * STAGE;
  const char* kimg = vimg + KEYS * Tile::ROWB;
  float* tab = reinterpret_cast<float*>(smem + 2 * STAGE + (VLDS + KLDS) * KEYS * Tile::ROWB);
  BiasSums<NW> sums;
  BiasSides sides;

  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), half = lane >> 5;
  const int nbk = a.B * a.kvh;
  const int ntile = cross_tiles(a.Sk, KEYS);
  const int bk = blockIdx.x % nbk, y = blockIdx.x / nbk;
  const int tile = y % ntile, part = y / ntile;  // causal: heaviest first
  const int b = bk / a.kvh, kv = bk % a.kvh;
  const int len = seq_len(a, b), start = seq_start(a, b);
  const int kw = wave % KW, qh = wave / KW;
  const int key0 = tile * KEYS, w0 = key0 + 32 * kw, j = w0 + (lane & 31);
  // query tiles that see the workgroup's keys, of each head of the group
  int first = 0;
  if (a.causal) first = max(0, key0 - start) / QT;
  int per = max(0, (a.Sq + QT - 1) / QT - first);
  if (key0 >= len || (a.causal && start + a.Sq <= key0)) per = 0;
  // the workgroup's tiles, over the heads of the group
  const int all = per * a.group;
  const int t0 = int(int64_t(all) * part / a.kv_parts);
  const int t1 = int(int64_t(all) * (part + 1) / a.kv_parts);

  const uint32_t lds0 = lds_addr(smem);
  // (tile of the head, head of the group) of the next copy and of this step,
  // counted along: divisions would be vector code
  struct Place {
    int i, h, per;
    __device__ __forceinline__ void step() {
      if (++i == per) {
        i = 0;
        ++h;
      }
    }
  };
  Place ahead{0, 0, per};
  if (t1 > t0) ahead = Place{t0 % per, t0 / per, per};
  Place now = ahead;
  auto issue = [&](int t) {
    const int h = kv * a.group + ahead.h, i0 = (first + ahead.i) * QT;
    ahead.step();
    const uint32_t to = lds0 + (t & 1) * STAGE;
    // queries in front of the first key: not read (0 x NaN would reach every key)
    const int low = a.causal ? -start - i0 : 0;
    Tile::template issue<QT, NW>(a.q.p + b * a.q.b + h * a.q.h + int64_t(i0) * a.q.t, a.q.t,
                                 a.Sq - i0, to, wave, lane, low);
    Tile::template issue<QT, NW>(a.dout.p + b * a.dout.b + h * a.dout.h + int64_t(i0) * a.dout.t,
                                 a.dout.t, a.Sq - i0, to + IMG, wave, lane, low);
    const int64_t at = (int64_t(b) * a.nh + h) * a.q_pad + i0;
    if (wave < 3) {  // (64 at a time; a 32-row tile uses half of them)
#pragma unroll
      for (int x = 0; x < NS; x += 64) {
        const int n = min(64, a.q_pad - i0 - x);  // the end of the rows: the last one again
        if (n > 0)
          dma4(rsrc_of((wave == 0 ? a.nlse : (wave == 1 ? a.ndelta : a.norm)) + at + x, 256),
               uni(to + 2 * IMG + wave * 4 * NS + 4 * x), uint32_t(min(lane, n - 1) * 4), 0u);
      }
    }
  };
  if (t1 > t0) {
    issue(t0);
    if constexpr (VLDS)
      Tile::template issue<KEYS, NW>(a.v.p + b * a.v.b + kv * a.v.h + int64_t(key0) * a.v.t,
                                     a.v.t, len - key0, lds0 + 2 * STAGE, wave, lane);
    if constexpr (KLDS)
      Tile::template issue<KEYS, NW>(a.k.p + b * a.k.b + kv * a.k.h + int64_t(key0) * a.k.t,
                                     a.k.t, len - key0, lds0 + 2 * STAGE + KEYS * Tile::ROWB, wave,
                                     lane);
  }

  typename Tile::RowFrag kf, vf;
  const int jc = max(0, min(j, len - 1));
  if (t1 > t0) {
    if constexpr (!KLDS)
      Tile::load_row(kf, a.k.p + b * a.k.b + kv * a.k.h + int64_t(jc) * a.k.t, half);
    if constexpr (!VLDS)
      Tile::load_row(vf, a.v.p + b * a.v.b + kv * a.v.h + int64_t(jc) * a.v.t, half);
  }
  floatx16 dk[Tile::ND], dv[Tile::ND];
#pragma unroll
  for (int d = 0; d < Tile::ND; ++d) {
    dk[d] = floatx16{};
    dv[d] = floatx16{};
  }
  // the bias gradient's sums of this workgroup's tiles of head h (of the group)
  auto sums_of = [&](int h) {
    const int64_t at = (int64_t(kv * a.group + h) * a.B + b) * ntile + tile;
    return a.dbias_part + (at * a.kv_parts + part) * a.bias.buckets;
  };
  if constexpr (BIAS) {
    sums.init(tab + bias_span(a.bias), a.bias, wave);
    for (int x = tid; x < a.group * a.bias.buckets; x += 64 * NW) {
      const int h = x / a.bias.buckets;
      if (t0 >= t1 || t0 >= (h + 1) * per || t1 <= h * per) sums_of(h)[x % a.bias.buckets] = 0.f;
    }
  }
  const float c = a.scale * LOG2E;
  for (int t = t0; t < t1; ++t, now.step()) {
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < t1) issue(t + 1);
    if constexpr (BIAS) {
      if (t == t0 || now.i == 0) {  // the next head (every wave is past the last one's tiles)
        if (t > t0) sums.flush(a.bias, sums_of(now.h - 1), tid, lane, wave);
        bias_spread(tab, a.bias, kv * a.group + now.h, a.nh, tid, 64 * NW);
        __syncthreads();
        sides.load(tab, a.bias);
        sums.clear(tid);
        __syncthreads();
      }
    }
    const int i0 = (first + now.i) * QT;
    if (w0 >= len || i0 + 32 * NB * qh >= a.Sq ||
        (a.causal && start + i0 + 32 * NB * (qh + 1) - 1 < w0))
      continue;
    const char* img = smem + (t & 1) * STAGE;
    const float* nls = reinterpret_cast<const float*>(img + 2 * IMG);
    const float* nds = nls + NS;
    const float* norms = nds + NS;
#pragma unroll
    for (int m = 0; m < NB; ++m) {
      const int n = qh * NB + m;
      floatx16 s = floatx16{}, dp;
      typename Tile::RowFrag af;
      if constexpr (KLDS) {
        Tile::rows(s, img, 32 * n, kimg, 32 * kw, lane);
      } else {
        Tile::load_rows(af, img, 32 * n, lane);
        issue_loads<AHEAD>();
        Tile::rows(s, af, kf);
      }
      if constexpr (!VLDS) Tile::load_rows(af, img + IMG, 32 * n, lane);
      // (fp32 reads it where it is used: it has no register left)
      float norm = 1.f;
      if constexpr (sizeof(T) == 2) norm = norms[32 * n + (lane & 31)];
      // (registers 4 q .. 4 q + 3: rows 8 q + 4 half on)
      const float* nlr = nls + 32 * n + 4 * half;
      const float* ndr = nds + 32 * n + 4 * half;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const floatx4 d = *reinterpret_cast<const floatx4*>(ndr + 2 * r);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[r + e] = d[e];
      }
      issue_loads<AHEAD>();
      if constexpr (VLDS)
        Tile::rows(dp, img + IMG, 32 * n, vimg, 32 * kw, lane);
      else
        Tile::rows(dp, af, vf);
      typename Tile::ColFrag cf;
      if constexpr (AHEAD) Tile::load_cols(cf, img + IMG, 32 * n, lane);
      issue_loads<AHEAD>();
      float ce = c, off = 0.f;
      int side = 0, at = 0;  // -1, 1: in a constant side, its entry taken apart
      if constexpr (BIAS) {
        const int tb = w0 - start - i0 - 32 * n;  // the block spans [tb - 31, tb + 31]
        side = sides.of(a.bias, tb - 31, tb + 31);
        if (side != 0) {
          off = sides.entry(side);
        } else {
          ce = 1.f;
          at = clampi(tb, a.bias.lo - 32, a.bias.hi + 32);  // (where the table has entries)
          const float* p = tab + (at + (lane & 31) - 4 * half - a.bias.lo + BIAS_PAD);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], c, p[-(8 * (r >> 2) + (r & 3))]);
        }
      }
      if (a.causal && start + i0 + 32 * n < w0 + 31) {
        // query start + i0 + 32 n + row sees key j from row = j - start - i0 - 32 n on
        const int from = j - start - i0 - 32 * n - 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) >= from ? s[r] : NEG_INF;
      }
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const floatx4 l = *reinterpret_cast<const floatx4*>(nlr + 2 * r);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[r + e] = exp2_hw(fmaf(s[r + e], ce, BIAS ? l[e] + off : l[e]));
      }
      if constexpr (sizeof(T) == 4) norm = norms[32 * n + (lane & 31)];
      if (__any(norm != 1.f)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= norms[32 * n + 4 * half + 8 * (r >> 2) + (r & 3)];
      }
      typename Tile::Probs p;
      Tile::pack(p, s);
      typename Tile::ColFrag qf;
      if constexpr (AHEAD) Tile::load_cols(qf, img, 32 * n, lane);
      if constexpr (!AHEAD) Tile::load_cols(cf, img + IMG, 32 * n, lane);
      Tile::cols(dv, cf, p, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= dp[r];
      if constexpr (BIAS) {
        // (a lane behind the sequence's keys holds what it read there)
        if (j >= len) s = floatx16{};
        if (side == 0) {
          sums.add(a.bias, s, at, lane);
        } else {
          float x = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) x += s[r];
          if (side < 0)
            sums.lo += x;
          else
            sums.hi += x;
        }
      }
      Tile::pack(p, s);
      if constexpr (!AHEAD) Tile::load_cols(qf, img, 32 * n, lane);
      Tile::cols(dk, qf, p, lane);
    }
  }
  if constexpr (BIAS) {
    if (t1 > t0) sums.flush(a.bias, sums_of((t1 - 1) / per), tid, lane, wave);
  }
  if constexpr (QH > 1) {
    // the others' sums to the first wave of the keys, one gradient after the other
    constexpr int BOX = 64 * 16 * Tile::ND;
    float* box = reinterpret_cast<float*>(smem) + lane;
    static_assert(KW * (QH - 1) * BOX * 4 <= 2 * STAGE, "the tiles' space holds a gradient");
    auto join = [&](floatx16(&x)[Tile::ND]) {
      __syncthreads();
      if (qh > 0) {
#pragma unroll
        for (int e = 0; e < 16 * Tile::ND; ++e) box[(wave - KW) * BOX + 64 * e] = x[e / 16][e % 16];
      }
      __syncthreads();
      if (qh == 0) {
#pragma unroll
        for (int k = 1; k < QH; ++k)
#pragma unroll
          for (int e = 0; e < 16 * Tile::ND; ++e)
            x[e / 16][e % 16] += box[(wave + (k - 1) * KW) * BOX + 64 * e];
      }
    };
    join(dk);
    join(dv);
    if (qh > 0) return;
  }
  // keys behind the sequence's length: zero
  const bool valid = j < a.Sk;
  if (j >= len) {
#pragma unroll
    for (int d = 0; d < Tile::ND; ++d) {
      dk[d] = floatx16{};
      dv[d] = floatx16{};
    }
  }
  if (a.kv_parts > 1) {
    const int64_t rows = int64_t(a.B) * a.kvh * a.Sk;
    const int64_t at = (part * rows + int64_t(bk) * a.Sk + j) * D;
    Tile::store_sums(a.part_dk + at, dk, valid, half);
    Tile::store_sums(a.part_dv + at, dv, valid, half);
    return;
  }
  Tile::store_row(a.dk.p + b * a.dk.b + kv * a.dk.h + int64_t(j) * a.dk.t, dk, a.scale, valid, half);
  Tile::store_row(a.dv.p + b * a.dv.b + kv * a.dv.h + int64_t(j) * a.dv.t, dv, 1.f, valid, half);
}

template <typename T, int D, bool BIAS, int NQ, int KS, int WV>
hipError_t run_q(const CrossArgs& a, hipStream_t s) {
  const size_t lds = cross_q_lds(sizeof(T), D, KS, BIAS ? bias_span_h(a.bias) : 0);
  hipError_t e = lds_limit<cross_bwd_q_kernel<T, D, BIAS, NQ, KS, WV>>(CROSS_LDS - 2048);
  if (e != hipSuccess) return e;
  const int64_t heads = int64_t(a.B) * a.nh;
  const int64_t grid = heads * cross_tiles(a.Sq, 32 * NQ) * a.q_parts;
  cross_bwd_q_kernel<T, D, BIAS, NQ, KS, WV><<<dim3(uint32_t(grid)), 64 * NQ * KS, lds, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess || a.q_parts == 1) return e;
  const int64_t n = heads * a.Sq * (D / 4);
  cross_join_q_kernel<T, D><<<dim3(uint32_t((n + 255) / 256)), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int D, bool BIAS, int KW, int QH>
hipError_t run_kv(const CrossArgs& a, hipStream_t s) {
  hipError_t e = lds_limit<cross_bwd_kv_kernel<T, D, BIAS, KW, QH>>(CROSS_LDS);
  if (e != hipSuccess) return e;
  const size_t lds = cross_kv_lds(sizeof(T), D, KW, QH, BIAS ? bias_span_h(a.bias) : 0);
  const int64_t heads = int64_t(a.B) * a.kvh;
  const int64_t grid = heads * cross_tiles(a.Sk, 32 * KW) * a.kv_parts;
  cross_bwd_kv_kernel<T, D, BIAS, KW, QH><<<dim3(uint32_t(grid)), 64 * KW * QH, lds, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int n = a.B * cross_tiles(a.Sk, 32 * KW) * a.kv_parts;
  if (a.kv_parts > 1) {
    const int64_t wgs = (heads * a.Sk * (D / 4) + 255) / 256;
    const dim3 grid(uint32_t(BIAS ? std::max<int64_t>(wgs, a.nh) : wgs), BIAS ? 3 : 2);
    cross_join_kv_kernel<T, D><<<grid, 256, 0, s>>>(a, n);
    return hipGetLastError();
  }
  if (!BIAS) return hipSuccess;
  cross_dbias_kernel<<<dim3(uint32_t(a.nh)), 256, 0, s>>>(a.dbias_part, a.dbias, n,
                                                          a.bias.buckets, a.nh);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_bwd_q(const CrossArgs& a, const CrossPlan& p, int dtype, int D,
                              hipStream_t s) {
  return cross_pick(dtype, D, a.bias.buckets > 0, [&](auto t, auto d, auto bias) {
    using T = typename decltype(t)::type;
    constexpr int DD = decltype(d)::value;
    constexpr bool BIAS = decltype(bias)::value;
    constexpr int WV = DD * sizeof(T) == 512 ? 1 : 2;
    if constexpr (DD * sizeof(T) < 512)
      if (p.q_split == 4) return run_q<T, DD, BIAS, 1, 4, WV>(a, s);
    if constexpr (cross_three(sizeof(T), DD))
      if (p.q_three)
        return p.q_split == 2 ? run_q<T, DD, BIAS, 2, 2, 3>(a, s)
                              : run_q<T, DD, BIAS, 4, 1, 3>(a, s);
    return p.q_split == 2 ? run_q<T, DD, BIAS, 2, 2, WV>(a, s) : run_q<T, DD, BIAS, 4, 1, WV>(a, s);
  });
}

hipError_t launch_cross_bwd_kv(const CrossArgs& a, const CrossPlan& p, int dtype, int D,
                               hipStream_t s) {
  return cross_pick(dtype, D, a.bias.buckets > 0, [&](auto t, auto d, auto bias) {
    using T = typename decltype(t)::type;
    constexpr int DD = decltype(d)::value;
    constexpr bool BIAS = decltype(bias)::value;
    if constexpr (cross_v_in_lds(sizeof(T), DD)) {
      if (p.kv_split == 4) return run_kv<T, DD, BIAS, 2, 4>(a, s);
      return p.kv_keys == 2 ? run_kv<T, DD, BIAS, 2, 2>(a, s) : run_kv<T, DD, BIAS, 4, 2>(a, s);
    } else {
      if constexpr (DD * sizeof(T) < 512)
        if (p.kv_split == 4) return run_kv<T, DD, BIAS, 1, 4>(a, s);
      return p.kv_split == 2 ? run_kv<T, DD, BIAS, 2, 2>(a, s) : run_kv<T, DD, BIAS, 4, 1>(a, s);
    }
  });
}

hipError_t launch_cross_no_keys(const CrossArgs& a, hipStream_t s) {
  cross_dbias_kernel<<<dim3(uint32_t(a.nh)), 256, 0, s>>>(a.dbias_part, a.dbias, 0, a.bias.buckets,
                                                          a.nh);
  return hipGetLastError();
}

}  // namespace abft
