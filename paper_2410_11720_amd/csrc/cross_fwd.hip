// Attention over keys of another length, forward.
//
// For query i of a sequence with n keys (n from k_lens), start = q_start:
//   s_ij = scale q_i . k_j + table[bucket(j - (start + i))],
//   o_i = sum_j softmax(s_i)_j v_j over j < n (and j <= start + i, causal),
// in one pass over the keys: with the running maximum m and sum l of a
// softmax in base 2, a tile adds p_j = 2^(s_ij log2 e - m) to l and
// p_j v_j to o; both are scaled when m grows by more than 2^8 (results do not
// depend on m, and 2^8 leaves fp32 sums far from overflow). A row without
// keys is zero and its lse minus infinity.
//
// Scores are formed as S^T = K Q^T, so that a lane holds the scores of one
// query (its row maximum and sum stay in the lane and its partner 32 lanes
// on) and P^T is the second operand of O^T = V^T P^T from registers.
#include "cross_tile.hpp"

namespace abft {
namespace {

// Longest distance that the running maximum may lag behind (log2 units).
constexpr float MAX_LAG = 8.f;

template <typename T, int D>
struct Online {
  using Tile = CrossTile<T, D>;
  floatx16 o[Tile::ND];
  float m, l;  // l: this lane's keys only

  __device__ __forceinline__ void init() {
    m = NEG_INF;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < Tile::ND; ++d) o[d] = floatx16{};
  }

  // One tile of NB x 32 keys: raw scores s (log2 score = s ce + off), their
  // values in the image v.
  template <int NB>
  __device__ __forceinline__ void add(floatx16 (&s)[NB], float ce, float off, const char* v,
                                      int lane) {
    typename Tile::ColFrag vf;
    Tile::load_cols(vf, v, 0, lane);
    issue_loads<sizeof(T) == 2>();
    float mt = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) mt = fmaxf(mt, s[b][r]);
    mt = fmaf(half_max(mt), ce, off);
    if (__any(mt > m + MAX_LAG)) {
      const float mn = fmaxf(m, mt);
      const float f = mn == NEG_INF ? 1.f : exp2_hw(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int d = 0; d < Tile::ND; ++d) o[d] *= f;
    }
    const float k = off - (m == NEG_INF ? 0.f : m);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = exp2_hw(fmaf(s[b][r], ce, k));
        l += s[b][r];
      }
      typename Tile::Probs p;
      Tile::pack(p, s[b]);
      typename Tile::ColFrag next;
      if (b + 1 < NB) Tile::load_cols(next, v, 32 * (b + 1), lane);
      Tile::cols(o, vf, p, lane);
      if (b + 1 < NB) vf = next;
    }
  }
};

// Scores of keys [at, at + 32) against the lane's query: keys from `limit`
// on (counted from `at`) are masked.
__device__ __forceinline__ void mask_scores(floatx16& s, int limit, int lane) {
  const int lim = limit - 4 * (lane >> 5);
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < lim ? s[r] : NEG_INF;
}

// Adds the spread bias to a block: s = s c + bias. p: the entry of the lane's
// query and the block's first key of the lane's half.
__device__ __forceinline__ void add_bias(floatx16& s, float c, const float* p) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], c, p[8 * (r >> 2) + (r & 3)]);
}

// Where the rest of an output row goes (null: nowhere; fp32 has none).
template <typename T, int D>
__device__ __forceinline__ char* rest_row(const CrossArgs& a, int b, int h, int i) {
  if (sizeof(T) == 4 || a.rest == nullptr) return nullptr;
  return a.rest + ((int64_t(b) * a.nh + h) * a.Sq + i) * D * 2;
}

// Tiled form: a workgroup owns 32 NQ queries of one head, KS waves for each 32 of
// them; key tiles pass through LDS in two stages, the next one copied while this
// one is worked on. The KS waves take different keys of a tile and join their
// sums at the end. Matrix cores are busy for 45% of its cycles at 4 x 2048 queries
// over 1024 keys, 32 heads on 8, head dim 128, the vector ALU for 50%: 171 us
// (median), 0.80 PFLOP/s of bf16. 8 x 1024 causal, 12 heads, head dim 64, with a
// bias: 24% and 56%, 28 us.
template <typename T, int D, bool BIAS, int NQ, int KS>
__global__ __launch_bounds__(64 * NQ * KS, 2) void cross_fwd_kernel(CrossArgs a) {
  using Tile = CrossTile<T, D>;
  constexpr int NW = NQ * KS, KT = cross_rows(sizeof(T), KS), NB = KT / 32 / KS;
  constexpr int IMG = KT * Tile::ROWB;
  extern __shared__ __align__(1024) char smem[];
  float* tab = reinterpret_cast<float*>(smem + 4 * IMG);

  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), half = lane >> 5;
  // sequences and key heads fastest: a head's tiles meet in one XCD's L2;
  // causal tiles heaviest first
  const int nbk = a.B * a.kvh;
  const int bk = blockIdx.x % nbk, y = blockIdx.x / nbk;
  const int b = bk / a.kvh, kv = bk % a.kvh, h = kv * a.group + y % a.group;
  int tile = y / a.group;
  if (a.causal) tile = cross_tiles(a.Sq, 32 * NQ) - 1 - tile;
  const int q0 = tile * 32 * NQ;
  const int len = seq_len(a, b), start = seq_start(a, b);
  int kend = len;
  if (a.causal) kend = min(kend, start + min(q0 + 32 * NQ, a.Sq));
  kend = max(kend, 0);
  const int nt = (kend + KT - 1) / KT;

  const int qw = wave % NQ, ks = wave / NQ;
  const int w0 = q0 + 32 * qw;               // the wave's first query
  const int i = w0 + (lane & 31);            // the lane's
  const bool valid = i < a.Sq;
  int wend = len;                            // keys of the wave
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
  if (nt > 0) issue(0);

  typename Tile::RowFrag q;
  Tile::load_row(q, a.q.p + b * a.q.b + h * a.q.h + int64_t(min(i, a.Sq - 1)) * a.q.t, half);
  if constexpr (BIAS) bias_spread(tab, a.bias, h, a.nh, tid, 64 * NW);
  BiasSides sides;

  Online<T, D> on;
  on.init();
  const float c = a.scale * LOG2E;
  for (int t = 0; t < nt; ++t) {
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < nt) issue(t + 1);
    if (BIAS && t == 0) sides.load(tab, a.bias);
    const int k0 = t * KT + 32 * NB * ks;    // the wave's keys of the tile
    if (k0 >= wend) continue;
    const char* img = smem + (t & 1) * 2 * IMG + 32 * NB * ks * Tile::ROWB;
    floatx16 s[NB];
    typename Tile::RowFrag kf[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) Tile::load_rows(kf[n], img, 32 * n, lane);
    issue_loads<sizeof(T) == 2>();
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      s[n] = floatx16{};
      Tile::rows(s[n], kf[n], q);
    }
    float ce = c, off = 0.f;
    if constexpr (BIAS) {
      // t of the corner; the wave's keys span [t0 - 31, t0 + 32 NB - 1]
      const int t0 = k0 - start - w0;
      if (const int side = sides.of(a.bias, t0 - 31, t0 + 32 * NB - 1)) {
        off = sides.entry(side);
      } else {
        ce = 1.f;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          // blocks of the tile may lie wholly in a constant side: t is
          // clamped to where the spread table has entries
          const int tb = clampi(t0 + 32 * n, a.bias.lo - 32, a.bias.hi + 32);
          add_bias(s[n], c, tab + (tb - (lane & 31) + 4 * half - a.bias.lo + BIAS_PAD));
        }
      }
    }
    if (k0 + 32 * NB > len || (a.causal && k0 + 32 * NB - 1 > start + w0)) {
#pragma unroll
      for (int n = 0; n < NB; ++n) mask_scores(s[n], limit - k0 - 32 * n, lane);
    }
    on.template add<NB>(s, ce, off, img + IMG, lane);
  }
  if constexpr (KS > 1) {
    // the others' maximum, sum and output to the first wave of the queries
    constexpr int BOX = 64 * (16 * Tile::ND + 2);
    float* box = reinterpret_cast<float*>(smem) + lane;
    static_assert(NQ * (KS - 1) * BOX * 4 <= 4 * IMG, "the tiles' space holds the boxes");
    __syncthreads();
    if (ks > 0) {
      float* p = box + (wave - NQ) * BOX;
      p[0] = on.m;
      p[64] = on.l;
#pragma unroll
      for (int e = 0; e < 16 * Tile::ND; ++e) p[64 * (e + 2)] = on.o[e / 16][e % 16];
    }
    __syncthreads();
    if (ks > 0) return;
#pragma unroll
    for (int k = 1; k < KS; ++k) {
      const float* p = box + (wave + (k - 1) * NQ) * BOX;
      // (a wave that saw no key adds nothing; one whose scores are all NaN has no
      // maximum either, but l = NaN)
      if (!__any(p[64] != 0.f)) continue;
      const float mk = p[0], mn = fmaxf(on.m, mk);
      const float f = mn == NEG_INF ? 1.f : exp2_hw(on.m - mn);
      const float g = mn == NEG_INF ? 0.f : exp2_hw(mk - mn);
      on.m = mn;
      on.l = fmaf(on.l, f, p[64] * g);
#pragma unroll
      for (int e = 0; e < 16 * Tile::ND; ++e)
        on.o[e / 16][e % 16] = fmaf(on.o[e / 16][e % 16], f, p[64 * (e + 2)] * g);
    }
  }
  const float l = half_sum(on.l);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  char* op = a.o.p + b * a.o.b + h * a.o.h + int64_t(i) * a.o.t;
  Tile::store_row(op, on.o, inv, valid, half, rest_row<T, D>(a, b, h, i));
  if (a.lse && valid && half == 0)
    a.lse[(int64_t(b) * a.nh + h) * a.Sq + i] = l == 0.f ? NEG_INF : on.m + log2_hw(l);
}

// Stages of the short form (fp32 rows of 128 elements leave room for one).
template <typename T, int D>
constexpr int short_stages() { return D * int(sizeof(T)) > 256 ? 1 : 2; }

// Short form, for few queries a sequence (decoded tokens): the queries of all
// heads that share a key head are one tile of up to 32 rows, the keys are
// split over workgroups and over the four waves of each. A wave copies
// its own 32-key tiles in two stages without workgroup barriers; the waves'
// results are joined in LDS, the splits' by cross_join_kernel. Bound by
// reading K and V (32 sequences of one query over up to 1500 keys, 32 heads, head
// dim 128: 116 us, 5.4 TB/s).
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(256) void cross_short_kernel(CrossArgs a) {
  using Tile = CrossTile<T, D>;
  constexpr int IMG = 32 * Tile::ROWB;
  constexpr int NS = short_stages<T, D>();
  constexpr int LDO = D + 4;
  extern __shared__ __align__(1024) char smem[];
  __shared__ float ml[4][32][2];
  __shared__ float side[32][2];             // bias of the constant sides, per row
  float* col = reinterpret_cast<float*>(smem + 8 * NS * IMG);               // [buckets][32]
  uint8_t* lut = reinterpret_cast<uint8_t*>(col + 32 * (BIAS ? a.bias.buckets : 0));

  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), half = lane >> 5;
  const int nbk = a.B * a.kvh, rows = a.Sq * a.group, ntile = (rows + 31) / 32;
  const int bk = blockIdx.x % nbk, y = blockIdx.x / nbk;
  const int b = bk / a.kvh, kv = bk % a.kvh;
  const int r0 = (y % ntile) * 32, split = y / ntile;
  const int len = seq_len(a, b), start = seq_start(a, b);
  const int row = min(r0 + (lane & 31), rows - 1);
  const int i = row / a.group, h = kv * a.group + row % a.group;
  const int i0 = r0 / a.group, i1 = min(r0 + 31, rows - 1) / a.group;
  int kend = len;
  if (a.causal) kend = min(kend, start + i1 + 1);
  kend = max(kend, 0);
  // this split's keys: whole steps of 128 (32 a wave)
  const int steps = (kend + 127) / 128, per = (steps + a.splits - 1) / a.splits;
  const int ks = split * per * 128, ke = min(kend, ks + per * 128);
  const int limit = a.causal ? min(len, start + i + 1) : len;
  int nt = 0;                                // the wave's 32-key tiles
  if (ks + 32 * wave < ke) nt = (ke - ks - 32 * wave + 127) / 128;

  const char* kp = a.k.p + b * a.k.b + kv * a.k.h;
  const char* vp = a.v.p + b * a.v.b + kv * a.v.h;
  char* mine = smem + wave * 2 * NS * IMG;
  const uint32_t lds0 = lds_addr(mine);
  auto issue = [&](int t) {
    const int k0 = ks + 32 * wave + 128 * t;
    const uint32_t to = lds0 + (t % NS) * 2 * IMG;
    Tile::template issue<32, 1>(kp + int64_t(k0) * a.k.t, a.k.t, len - k0, to, 0, lane);
    Tile::template issue<32, 1>(vp + int64_t(k0) * a.v.t, a.v.t, len - k0, to + IMG, 0, lane);
  };
  constexpr int RUNS = 2 * 32 / Tile::RPR;   // copies a stage
  typename Tile::RowFrag q;
  Tile::load_row(q, a.q.p + b * a.q.b + h * a.q.h + int64_t(i) * a.q.t, half);
  if (nt > 0) issue(0);
  if (NS > 1 && nt > 1) issue(1);
  bool lo_apart = true, hi_apart = true;
  if constexpr (BIAS) {
    const int n = a.bias.hi - a.bias.lo + 1;
    for (int x = tid; x < n; x += 256) lut[x] = uint8_t(bias_bucket(a.bias, x + a.bias.lo));
    for (int x = tid; x < 32 * a.bias.buckets; x += 256) {
      const int g = kv * a.group + min(r0 + (x & 31), rows - 1) % a.group;
      col[x] = bias_entry(a.bias.table[int64_t(x >> 5) * a.nh + g]);
    }
    __syncthreads();
    if (tid < 64)
      side[tid & 31][tid >> 5] = col[32 * lut[tid < 32 ? 0 : n - 1] + (tid & 31)];
    __syncthreads();
    lo_apart = __all(side_apart(side[lane & 31][0]));
    hi_apart = __all(side_apart(side[lane & 31][1]));
  }

  Online<T, D> on;
  on.init();
  const float c = a.scale * LOG2E;
  for (int t = 0; t < nt; ++t) {
    if (NS > 1 && t + 1 < nt)
      wait_vmcnt<RUNS>();
    else
      wait_vmcnt<0>();
    __builtin_amdgcn_wave_barrier();
    const int k0 = ks + 32 * wave + 128 * t;
    const char* img = mine + (t % NS) * 2 * IMG;
    floatx16 s[1] = {floatx16{}};
    typename Tile::RowFrag kf;
    Tile::load_rows(kf, img, 0, lane);
    issue_loads<sizeof(T) == 2>();
    Tile::rows(s[0], kf, q);
    float ce = c, off = 0.f;
    if constexpr (BIAS) {
      const int lo = a.bias.lo, hi = a.bias.hi;
      if (lo_apart && k0 + 31 - start - i0 <= lo) {
        off = side[lane & 31][0];
      } else if (hi_apart && k0 - start - i1 >= hi) {
        off = side[lane & 31][1];
      } else {
        ce = 1.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int t1 = k0 + 8 * (r >> 2) + 4 * half + (r & 3) - start - i;
          s[0][r] = fmaf(s[0][r], c, col[32 * lut[clampi(t1, lo, hi) - lo] + (lane & 31)]);
        }
      }
    }
    if (k0 + 32 > len || a.causal) mask_scores(s[0], limit - k0, lane);
    on.template add<1>(s, ce, off, img + IMG, lane);
    if (t + NS < nt) {
      lds_wait_all();  // the stage has been read
      issue(t + NS);
    }
  }

  // join the waves (their tiles have landed and been read)
  const float l = half_sum(on.l);
  __syncthreads();
  float* ob = reinterpret_cast<float*>(smem);  // [4][32][LDO]
  if (half == 0) {
    ml[wave][lane][0] = on.m;
    ml[wave][lane][1] = l;
  }
  if (nt > 0) {
    float* p = ob + (wave * 32 + (lane & 31)) * LDO;
#pragma unroll
    for (int d = 0; d < Tile::ND; ++d)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<floatx4*>(p + 32 * d + 8 * k + 4 * half) =
            floatx4{on.o[d][4 * k], on.o[d][4 * k + 1], on.o[d][4 * k + 2], on.o[d][4 * k + 3]};
  }
  __syncthreads();
  constexpr int TPR = 8, PER = D / TPR;      // threads a row, elements a thread
  const int jr = tid / TPR, j0 = (tid % TPR) * PER;
  if (r0 + jr >= rows) return;
  float mm = NEG_INF;
#pragma unroll
  for (int w = 0; w < 4; ++w) mm = fmaxf(mm, ml[w][jr][0]);
  float acc[PER] = {}, lt = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float lw = ml[w][jr][1];
    if (lw == 0.f) continue;                 // no key seen: its sums are not written
    const float f = exp2_hw(ml[w][jr][0] - mm);
    lt = fmaf(lw, f, lt);
#pragma unroll
    for (int e = 0; e < PER; ++e)
      acc[e] = fmaf(ob[(w * 32 + jr) * LDO + j0 + e], f, acc[e]);
  }
  const int out_row = r0 + jr;
  if (a.splits == 1) {
    const int oi = out_row / a.group, oh = kv * a.group + out_row % a.group;
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    char* op = a.o.p + b * a.o.b + oh * a.o.h + int64_t(oi) * a.o.t + j0 * int(sizeof(T));
    char* rp = rest_row<T, D>(a, b, oh, oi);
#pragma unroll
    for (int e = 0; e < PER; e += 4) {
      const floatx4 x = {acc[e] * inv, acc[e + 1] * inv, acc[e + 2] * inv, acc[e + 3] * inv};
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<u32x2*>(op + e * 2) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
        if (rp != nullptr)
          *reinterpret_cast<u32x2*>(rp + (j0 + e) * 2) =
              u32x2{pack_bf16(rounding_rest(x[0]), rounding_rest(x[1])),
                    pack_bf16(rounding_rest(x[2]), rounding_rest(x[3]))};
      } else {
        *reinterpret_cast<floatx4*>(op + e * 4) = x;
      }
    }
    if (a.lse && j0 == 0)
      a.lse[(int64_t(b) * a.nh + oh) * a.Sq + oi] = lt == 0.f ? NEG_INF : mm + log2_hw(lt);
  } else {
    const int64_t at = (int64_t(bk) * rows + out_row) * a.splits + split;
    if (j0 == 0) {
      a.part_ml[2 * at] = mm;
      a.part_ml[2 * at + 1] = lt;
    }
    if (lt != 0.f) {
#pragma unroll
      for (int e = 0; e < PER; e += 4)
        *reinterpret_cast<floatx4*>(a.part_o + at * D + j0 + e) =
            floatx4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
    }
  }
}

// Joins the splits of the short form, at most 64: a wave per row. Lane s holds
// split s's maximum and sum; the outputs are read four splits at a time and
// summed in the order of the splits (a split that saw no key wrote none).
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossArgs a) {
  const int lane = threadIdx.x & 63;
  const int rows = a.Sq * a.group;
  const int64_t r = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (r >= int64_t(a.B) * a.kvh * rows) return;
  const bool in = lane < a.splits;
  const float* ml = a.part_ml + (r * a.splits + (in ? lane : 0)) * 2;
  const float ls = in ? ml[1] : 0.f, ms = in && ls != 0.f ? ml[0] : NEG_INF;
  float m = ms;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
  const float f = ls != 0.f ? exp2_hw(ms - m) : 0.f;
  const float l = group_sum<64>(ls * f);
  constexpr int PER = D / 64, U = 4;
  typedef float vec __attribute__((ext_vector_type(PER)));
  const vec* po = reinterpret_cast<const vec*>(a.part_o + r * a.splits * D) + lane;
  vec acc = {};
  for (int s = 0; s < a.splits; s += U) {
    vec x[U];
    float w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = min(s + u, a.splits - 1);
      x[u] = po[at * 64];
      w[u] = __shfl(f, at, 64);
      if (s + u >= a.splits) w[u] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (w[u] != 0.f) acc += x[u] * w[u];
  }
  const int bk = int(r / rows), row = int(r % rows);
  const int b = bk / a.kvh, h = (bk % a.kvh) * a.group + row % a.group, i = row / a.group;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* op = reinterpret_cast<T*>(a.o.p + b * a.o.b + h * a.o.h + int64_t(i) * a.o.t) + lane * PER;
  T* rp = reinterpret_cast<T*>(rest_row<T, D>(a, b, h, i));
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    op[e] = Storage<T>::store(acc[e] * inv);
    if (rp != nullptr) rp[lane * PER + e] = Storage<T>::store(rounding_rest(acc[e] * inv));
  }
  if (a.lse && lane == 0)
    a.lse[(int64_t(b) * a.nh + h) * a.Sq + i] = l == 0.f ? NEG_INF : m + log2_hw(l);
}

template <typename T, int D, bool BIAS, int NQ, int KS>
hipError_t run_fwd(const CrossArgs& a, hipStream_t s) {
  const size_t lds = cross_q_lds(sizeof(T), D, KS, BIAS ? bias_span_h(a.bias) : 0);
  hipError_t e = lds_limit<cross_fwd_kernel<T, D, BIAS, NQ, KS>>(CROSS_LDS);
  if (e != hipSuccess) return e;
  const int64_t grid = int64_t(a.B) * a.nh * cross_tiles(a.Sq, 32 * NQ);
  cross_fwd_kernel<T, D, BIAS, NQ, KS><<<dim3(uint32_t(grid)), 64 * NQ * KS, lds, s>>>(a);
  return hipGetLastError();
}

template <typename T, int D, bool BIAS>
hipError_t run_short(const CrossArgs& a, hipStream_t s) {
  size_t lds = size_t(8) * short_stages<T, D>() * 32 * D * sizeof(T);
  if (BIAS) lds += size_t(a.bias.buckets) * 128 + size_t(a.bias.hi - a.bias.lo + 1);
  hipError_t e = lds_limit<cross_short_kernel<T, D, BIAS>>(158 * 1024);
  if (e != hipSuccess) return e;
  const int rows = a.Sq * a.group;
  const int64_t grid = int64_t(a.B) * a.kvh * ((rows + 31) / 32) * a.splits;
  cross_short_kernel<T, D, BIAS><<<dim3(uint32_t(grid)), 256, lds, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess || a.splits == 1) return e;
  const int64_t n = int64_t(a.B) * a.kvh * rows;
  cross_join_kernel<T, D><<<dim3(uint32_t((n + 3) / 4)), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_fwd(const CrossArgs& a, int dtype, int D, hipStream_t s) {
  return cross_pick(dtype, D, a.bias.buckets > 0, [&](auto t, auto d, auto bias) {
    using T = typename decltype(t)::type;
    constexpr int D = decltype(d)::value;
    constexpr bool BIAS = decltype(bias)::value;
    const int64_t heads = int64_t(a.B) * a.nh, blocks = cross_tiles(a.Sk, 32);
    const int most = sizeof(T) * D == 128 ? 3 : 2, span = BIAS ? bias_span_h(a.bias) : 0;
    auto lds = [&](int split) { return cross_q_lds(sizeof(T), D, split, span); };
    if constexpr (D * sizeof(T) < 512)  // (four 32-row tiles of 512 bytes do not fit LDS)
      if (cross_split_pays(4, heads * cross_tiles(a.Sq, 32), lds(4), most, blocks, int(sizeof(T))))
        return run_fwd<T, D, BIAS, 1, 4>(a, s);
    if (cross_split_pays(2, heads * cross_tiles(a.Sq, 64), lds(2), most, blocks, int(sizeof(T))))
      return run_fwd<T, D, BIAS, 2, 2>(a, s);
    return run_fwd<T, D, BIAS, 4, 1>(a, s);
  });
}

hipError_t launch_cross_short(const CrossArgs& a, int dtype, int D, hipStream_t s) {
  return cross_pick(dtype, D, a.bias.buckets > 0, [&](auto t, auto d, auto bias) {
    return run_short<typename decltype(t)::type, decltype(d)::value, decltype(bias)::value>(a, s);
  });
}

}  // namespace abft
