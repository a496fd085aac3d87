// Descriptors of the attention kernels over keys of another length, shared
// by the kernels and the host entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "abft_internal.hpp"

namespace abft {

// One operand: rows of head_dim elements, strides in bytes.
struct CrossTensor {
  char* p = nullptr;
  int64_t b = 0, h = 0;  // between sequences, between heads
  uint32_t t = 0;        // between tokens
};

constexpr int CROSS_MAX_BUCKETS = 128;
constexpr int CROSS_MAX_DISTANCE = 1024;

// Relative position bias: bucket of t = key - query position (see
// attn_rel_bucket). t <= lo and t >= hi have one bucket each.
struct CrossBias {
  const float* table = nullptr;  // [buckets][heads]
  int buckets = 0, bidirectional = 0;
  int side = 0;   // buckets of one side
  int exact = 0;  // of them, distances with a bucket of their own
  int lo = 0, hi = 0;
  int32_t border[CROSS_MAX_BUCKETS];  // [i], i >= 1: least distance of bucket exact + i
};

struct CrossArgs {
  int B = 0, Sq = 0, Sk = 0, nh = 0, kvh = 0, group = 1;
  int causal = 0;
  float scale = 1.f;
  CrossTensor q, k, v, o;                  // forward: o written; backward: read
  CrossTensor dout, dq, dk, dv;            // backward
  const int32_t* k_lens = nullptr;         // [B] or null
  const int32_t* q_start = nullptr;        // [B] or null
  float* lse = nullptr;                    // [B][nh][Sq], base 2; may be null forward
  char* rest = nullptr;                    // [B][nh][Sq][D]: what rounding took off O; may be null
  // short form: key splits and their partial results
  int splits = 1;
  float* part_o = nullptr;                 // [B][kvh][rows][splits][D]
  float* part_ml = nullptr;                // [B][kvh][rows][splits][2]
  // backward
  int q_pad = 0;                           // Sq rounded up to the query tile
  float* nlse = nullptr;                   // [B][nh][q_pad]: -lse (-inf: no key)
  float* ndelta = nullptr;                 // [B][nh][q_pad]: -D
  float* norm = nullptr;                   // [B][nh][q_pad]: 1 / sum of the row's 2^(s - lse)
  float* dbias_part = nullptr;             // [nh][B * key tiles * kv_parts][buckets]
  // the passes' other axis split over workgroups, and the parts' results
  int q_parts = 1, kv_parts = 1;
  float* part_dq = nullptr;                // [q_parts][B][nh][Sq][D]
  float* part_sum = nullptr;               // [q_parts][B][nh][q_pad]
  float* part_dk = nullptr;                // [kv_parts][B][kvh][Sk][D]
  float* part_dv = nullptr;
  float* dbias = nullptr;                  // [buckets][nh]
  CrossBias bias;
};

constexpr int CROSS_QT = 128;  // queries (keys) a workgroup owns at most in the tiled kernels

constexpr int cross_tiles(int n, int tile) { return (n + tile - 1) / tile; }

constexpr size_t CROSS_LDS = 160 * 1024;

// Rows of a tile of the other axis, for `split` waves that share it (es: bytes of
// an element), and entries of their statistics in LDS (copied 64 at a time).
constexpr int cross_rows(int es, int split) {
  return std::max(es == 2 ? 64 : 32, 32 * split);
}
constexpr int cross_stats(int rows) { return std::max(64, rows); }

// LDS of a workgroup: two stages of two images (forward, query pass); in the
// key pass the statistics too, for bf16 rows of 256 bytes the values (and with a
// bias the keys, which leaves its registers for the diagonal sums), and the sums of
// the bias gradient.
constexpr size_t cross_q_lds(int es, int D, int split, int span) {
  return size_t(4) * cross_rows(es, split) * D * es + size_t(span) * 4;
}
constexpr bool cross_v_in_lds(int es, int D) { return es == 2 && D == 128; }
constexpr bool cross_k_in_lds(int es, int D, int QH, bool bias) {
  return cross_v_in_lds(es, D) && bias && QH == 2;
}
constexpr size_t cross_kv_lds(int es, int D, int KW, int QH, int span) {
  return 2 * (size_t(2) * cross_rows(es, QH) * D * es + 12 * cross_stats(cross_rows(es, QH))) +
         (cross_v_in_lds(es, D) ? size_t(32) * KW * D * es : 0) +
         (cross_k_in_lds(es, D, QH, span > 0) ? size_t(32) * KW * D * es : 0) +
         size_t(span ? KW * QH + 1 : 0) * span * 4;
}

// Whether `split` waves (2 or 4) share the work of 32 queries (keys), each a part
// of the other axis: where all workgroups of that shape are on the chip at once.
// A wave's tiles follow each other, and fewer than two waves a SIMD leave its
// waits uncovered, so a grid that does not fill the chip gains (8 heads, 1024
// queries and keys: 67 -> 35 us by 4; fp32 374 -> 121 us); one that does loses what
// the smaller tiles read twice (16 heads x 4096: 345 -> 449 us).
// wgs: workgroups of the shape; lds: bytes each takes; most: that a CU's
// registers hold; blocks: 32s along the split axis. In bf16 each wave needs two of
// them to make up for the join; in fp32, with matrix cores at a sixteenth of the
// rate, one will do (2 x 128 over 96, 8 heads of 64: forward and backward 45 -> 37
// us; in bf16 8 x 64 over 64, 16 heads, takes 17 us, split 19).
inline bool cross_split_pays(int split, int64_t wgs, size_t lds, int most, int64_t blocks,
                             int es) {
  if (lds > CROSS_LDS || blocks < (es == 4 ? split : 2 * split)) return false;
  return wgs <= 256 * std::min<int64_t>(most, int64_t(CROSS_LDS / lds));
}

// Over how many workgroups the other axis is split, each leaving fp32 sums that a
// further launch joins: as many as fill the chip, where that saves more steps (tiles
// one after the other, about 1 us) than the launch and the sums cost.
inline int cross_parts(int64_t wgs, size_t lds, int most, int64_t steps, int64_t cost) {
  const int64_t slots = 256 * std::min<int64_t>(most, int64_t(CROSS_LDS / lds));
  const int64_t n = std::min<int64_t>({16, slots / std::max<int64_t>(wgs, 1), steps / 2});
  return n > 1 && steps - (steps + n - 1) / n > cost ? int(n) : 1;
}

// Whether the query pass has a form with fewer registers, three workgroups to a
// CU. It takes grids that two a CU do not hold at once (cross attention of 8 x
// 512 over 1000, 12 heads: both passes in 6% less; 2 x 4096, 32 heads: 2%); a
// grid that two a CU hold is better off with fragments read ahead (16 heads x
// 4096: in three 2% more).
constexpr bool cross_three(int es, int D) { return es * D == 128; }

// Shapes of the backward passes.
struct CrossPlan {
  int q_split = 1, q_parts = 1;    // waves, workgroups that share 32 queries
  bool q_three = false;            // three workgroups of the query pass a CU, not two
  int kv_keys = 4, kv_split = 1;   // 32s of keys of a workgroup, waves that share 32 keys
  int kv_parts = 1;
};
inline CrossPlan cross_plan(int64_t B, int nh, int kvh, int64_t Sq, int64_t Sk, int es, int D,
                            int span) {
  CrossPlan p;
  const bool wide = D * es == 512;  // (four 32-row tiles of 512 bytes do not fit LDS)
  const int64_t qh = B * nh, kh = B * kvh;
  const int64_t sq = cross_tiles(int(Sq), 32), sk = cross_tiles(int(Sk), 32);
  const int64_t cost = es == 4 ? 1 : 4;
  const int most = wide ? 1 : 2;
  if (!wide && cross_split_pays(4, qh * sq, cross_q_lds(es, D, 4, span), most, sk, es))
    p.q_split = 4;
  else if (cross_split_pays(2, qh * ((sq + 1) / 2), cross_q_lds(es, D, 2, span),
                            cross_three(es, D) ? 3 : most, sk, es))
    p.q_split = 2;
  const int64_t wgs = qh * cross_tiles(int(sq), 4 / p.q_split);
  p.q_three = cross_three(es, D) && wgs > 256 * most;
  p.q_parts = cross_parts(wgs, cross_q_lds(es, D, p.q_split, span), most,
                          cross_tiles(int(Sk), cross_rows(es, p.q_split)), cost);
  const int64_t blocks = nh / kvh * sq, two = kh * ((sk + 1) / 2);
  if (cross_v_in_lds(es, D)) {
    // (8 waves a workgroup, and a CU; the sums of a wide bias leave room for 4)
    p.kv_split = 2;
    if (cross_split_pays(4, two, cross_kv_lds(es, D, 2, 4, span), 1, blocks, es)) {
      p.kv_keys = 2;
      p.kv_split = 4;
    } else if (cross_kv_lds(es, D, 4, 2, span) > CROSS_LDS) {
      p.kv_keys = 2;
    }
  } else if (!wide &&
             cross_split_pays(4, kh * sk, cross_kv_lds(es, D, 1, 4, span), most, blocks, es)) {
    p.kv_keys = 1;
    p.kv_split = 4;
  } else if (cross_split_pays(2, two, cross_kv_lds(es, D, 2, 2, span), most, blocks, es)) {
    p.kv_keys = p.kv_split = 2;
  }
  const int64_t heads = nh / kvh;
  // (a head's bias gradient is joined when the workgroup leaves the head: three steps)
  p.kv_parts = cross_parts(kh * cross_tiles(int(sk), p.kv_keys),
                           cross_kv_lds(es, D, p.kv_keys, p.kv_split, span),
                           p.kv_keys * p.kv_split > 4 ? 1 : most,
                           heads * cross_tiles(int(Sq), cross_rows(es, p.kv_split)) +
                               (span ? 3 * heads : 0),
                           cost);
  return p;
}

// Entries of the spread bias table in LDS.
constexpr int CROSS_BIAS_PAD = 63;
inline int bias_span_h(const CrossBias& b) { return b.hi - b.lo + 1 + 2 * CROSS_BIAS_PAD; }

template <typename T> struct TypeTag { using type = T; };

// Calls f with tags of the storage type, head dim and presence of a bias.
template <typename F>
hipError_t cross_pick(int dtype, int D, bool bias, F f) {
  auto by_bias = [&](auto t, auto d) {
    return bias ? f(t, d, std::true_type{}) : f(t, d, std::false_type{});
  };
  auto by_dim = [&](auto t) {
    return D == 64 ? by_bias(t, std::integral_constant<int, 64>{})
                   : by_bias(t, std::integral_constant<int, 128>{});
  };
  return dtype == ABFT_FP32 ? by_dim(TypeTag<float>{}) : by_dim(TypeTag<uint16_t>{});
}

hipError_t launch_cross_fwd(const CrossArgs& a, int dtype, int D, hipStream_t s);
hipError_t launch_cross_short(const CrossArgs& a, int dtype, int D, hipStream_t s);
hipError_t launch_cross_bwd_q(const CrossArgs& a, const CrossPlan& p, int dtype, int D,
                              hipStream_t s);
hipError_t launch_cross_bwd_kv(const CrossArgs& a, const CrossPlan& p, int dtype, int D,
                               hipStream_t s);
hipError_t launch_cross_no_keys(const CrossArgs& a, hipStream_t s);  // a bias gradient of zeros

}  // namespace abft
