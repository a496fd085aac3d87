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
  float* dbias_part = nullptr;             // [nh][B * key tiles][buckets]
  float* dbias = nullptr;                  // [buckets][nh]
  CrossBias bias;
};

constexpr int CROSS_QT = 128;  // queries (keys) a workgroup owns at most in the tiled kernels
constexpr int CROSS_QMIN = 32;  // and at least

constexpr int cross_tiles(int n, int tile) { return (n + tile - 1) / tile; }

constexpr size_t CROSS_LDS = 160 * 1024;

// Whether `split` waves (2 or 4) share the work of 32 queries (keys), each a part
// of the other axis: where all workgroups of that shape are on the chip at once. A wave's tiles follow each other, and fewer than two waves a
// SIMD leave its waits uncovered, so a grid that does not fill the chip gains
// (8 heads, 1024 queries and keys: 67 -> 35 us by 4; fp32 374 -> 121 us); one that
// does loses what the smaller tiles read twice (16 heads x 4096: 345 -> 449 us).
// wgs: workgroups of the shape; lds: bytes each takes; most: that a CU's
// registers hold; blocks: 32s along the split axis.
inline bool cross_split_pays(int split, int64_t wgs, size_t lds, int most, int64_t blocks) {
  if (lds > CROSS_LDS || blocks < 2 * split) return false;
  return wgs <= 256 * std::min<int64_t>(most, int64_t(CROSS_LDS / lds));
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
hipError_t launch_cross_bwd_q(const CrossArgs& a, int dtype, int D, hipStream_t s);
hipError_t launch_cross_bwd_kv(const CrossArgs& a, int dtype, int D, hipStream_t s);
hipError_t launch_cross_no_keys(const CrossArgs& a, hipStream_t s);  // a bias gradient of zeros

}  // namespace abft
