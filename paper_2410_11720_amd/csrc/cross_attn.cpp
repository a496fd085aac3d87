// Host entry points of attention over keys of another length
// (include/attn_abft.h): checks, workspace layout, choice of the form.
#include <algorithm>
#include <cmath>

#include "cross_internal.hpp"
#include "overlap.hpp"

namespace abft {
namespace {

constexpr size_t ALIGN = 256;
constexpr int MAX_LEN = 1 << 29;             // positions and their differences fit 32 bits
constexpr int64_t MAX_TOKEN_BYTES = 1 << 24; // a tile's rows fit the copies' 32-bit offsets
constexpr int64_t MAX_EXTENT = int64_t(1) << 56;  // bytes between a dimension's ends

size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
int es_of(const attn_cross_config* c) { return c->dtype == ABFT_FP32 ? 4 : 2; }

// Least whole n with n >= e (m / e)^(t / f), i.e. n^f >= e^(f - t) m^t: exact.
// Where the right side lies within 1e-9 of a whole number, that number's prime
// exponents tell whether both sides are equal; else extended precision decides.
int border(int e, int m, int t, int f) {
  const double x = e * std::pow(double(m) / e, double(t) / f);
  const double near = std::round(x);
  if (std::fabs(x - near) > 1e-9 * x) return int(std::ceil(x));
  int a = int(near), b = e, c = m;
  bool equal = true;
  for (int p = 2; a > 1 || b > 1 || c > 1; ++p) {
    int va = 0, vb = 0, vc = 0;
    while (a % p == 0) { a /= p; ++va; }
    while (b % p == 0) { b /= p; ++vb; }
    while (c % p == 0) { c /= p; ++vc; }
    equal = equal && f * va == (f - t) * vb + t * vc;
  }
  const long double l = f * std::log((long double)near), r = (f - t) * std::log((long double)e) +
                                                             t * std::log((long double)m);
  return int(near) + (equal || l > r ? 0 : 1);
}

bool make_bias(int buckets, int max_distance, int bidirectional, CrossBias* b) {
  if (buckets > CROSS_MAX_BUCKETS || max_distance > CROSS_MAX_DISTANCE) return false;
  if (bidirectional != 0 && bidirectional != 1) return false;
  if (bidirectional && buckets % 2) return false;
  b->buckets = buckets;
  b->bidirectional = bidirectional;
  b->side = bidirectional ? buckets / 2 : buckets;
  if (b->side < 2) return false;
  b->exact = b->side / 2;
  if (max_distance <= b->exact) return false;
  const int f = b->side - b->exact;
  b->border[0] = b->exact;
  for (int t = 1; t < f; ++t) b->border[t] = border(b->exact, max_distance, t, f);
  b->lo = -b->border[f - 1];
  b->hi = bidirectional ? b->border[f - 1] : 0;
  return true;
}

int validate(const attn_cross_config* c, CrossBias* bias) {
  if (!c || c->batch < 0 || c->q_len < 0 || c->k_len < 0 || c->heads < 1 || c->kv_heads < 1)
    return ABFT_ERR_INVALID;
  if (c->heads % c->kv_heads) return ABFT_ERR_INVALID;
  if (c->causal != 0 && c->causal != 1) return ABFT_ERR_INVALID;
  if (!std::isfinite(c->scale)) return ABFT_ERR_INVALID;
  if (c->buckets < 0) return ABFT_ERR_INVALID;
  if (c->dtype != ABFT_BF16 && c->dtype != ABFT_FP32) return ABFT_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return ABFT_ERR_UNSUPPORTED;
  if (c->q_len > MAX_LEN || c->k_len > MAX_LEN) return ABFT_ERR_UNSUPPORTED;
  const int64_t wgs = int64_t(c->batch) * c->heads;
  if (wgs > (int64_t(1) << 24) ||
      wgs * cross_tiles(std::max(c->q_len, c->k_len), 32) > (int64_t(1) << 30))
    return ABFT_ERR_UNSUPPORTED;
  if (c->buckets && !make_bias(c->buckets, c->max_distance, c->bidirectional, bias))
    return ABFT_ERR_INVALID;
  return ABFT_OK;
}

// Whether the short form takes a forward, and its key splits, by the steps (128
// keys, a wave 32 of them) that follow each other on a CU. The short form runs the
// queries of all heads that share a key head as tiles of 32 rows and may
// split the keys over workgroups, which costs a second launch (about 3 us, a
// step 0.65 us at head dim 64 and 1 us at 128); the tiled form runs every
// 32 queries of a head over all keys. Measured: 8 heads x 2 sequences, 32 queries
// over 2000 keys, head dim 64: 9.5 us, tiled 14.5; 12 x 16, 500 keys: tiled
// 7.8, two splits 13.1.
bool short_form(const attn_cross_config* c, int* splits) {
  *splits = 1;
  const int64_t row = int64_t(c->head_dim) * es_of(c);     // bytes
  const int64_t rows = int64_t(c->q_len) * (c->heads / c->kv_heads);
  const int64_t base = int64_t(c->batch) * c->kv_heads * ((rows + 31) / 32);
  if (base == 0 || rows > 65536) return false;
  const int64_t steps = (int64_t(c->k_len) + 127) / 128;
  const int64_t slots = row == 128 ? 512 : 256;            // workgroups at a time, by LDS
  const int64_t join = es_of(c) == 4 ? 1 : (row == 128 ? 5 : 4);
  const int64_t most = std::min<int64_t>({64, steps / 2, slots / base});
  int64_t cost = (base + slots - 1) / slots * steps;
  if (most > 1 && (steps + most - 1) / most + join < cost) {
    *splits = int(most);
    cost = (steps + most - 1) / most + join;
  }
  const int64_t tiles = int64_t(c->batch) * c->heads * cross_tiles(c->q_len, 32);
  const int64_t tiled = std::max(steps, tiles * steps / slots);
  return cost < tiled || (cost == tiled && rows <= 32);
}

struct Space {
  size_t part_o = 0, part_ml = 0;        // forward, short form
  size_t nlse = 0, ndelta = 0, norm = 0, dbias = 0;  // backward
  size_t sum = 0, part = 0, part2 = 0;               // its parts (one pass's at a time)
  size_t fwd = 0, bwd = 0;
};

CrossPlan plan_of(const attn_cross_config* c, const CrossBias& b) {
  return cross_plan(c->batch, c->heads, c->kv_heads, c->q_len, c->k_len, es_of(c), c->head_dim,
                    c->buckets ? bias_span_h(b) : 0);
}

Space make_space(const attn_cross_config* c, const CrossPlan& p) {
  Space L;
  int splits;
  if (short_form(c, &splits) && splits > 1) {
    const size_t n = size_t(c->batch) * c->heads * c->q_len * splits;
    L.part_o = 0;
    L.part_ml = align_up(n * c->head_dim * 4);
    L.fwd = L.part_ml + align_up(n * 8);
  }
  const size_t rows = size_t(c->batch) * c->heads * cross_tiles(c->q_len, CROSS_QT) * CROSS_QT;
  L.ndelta = align_up(rows * 4);
  L.norm = 2 * L.ndelta;
  L.dbias = 3 * L.ndelta;
  L.sum = L.dbias + align_up(size_t(c->batch) * c->heads * cross_tiles(c->k_len, 32 * p.kv_keys) *
                             p.kv_parts * c->buckets * 4);
  L.part = L.sum + (p.q_parts > 1 ? align_up(rows * 4 * p.q_parts) : 0);
  const size_t dq = size_t(c->batch) * c->heads * c->q_len * c->head_dim * 4;
  const size_t dk =
      align_up(size_t(c->batch) * c->kv_heads * c->k_len * c->head_dim * 4 * p.kv_parts);
  L.part2 = L.part + dk;
  L.bwd = L.part + std::max(p.q_parts > 1 ? align_up(dq * p.q_parts) : 0,
                            p.kv_parts > 1 ? 2 * dk : 0);
  return L;
}

// An operand as the kernels take it: n tokens of nh heads.
int take(const attn_cross_config* c, const attn_cross_tensor* t, int n, int nh, bool out,
         CrossTensor* r) {
  if (!t) return ABFT_ERR_INVALID;
  if (c->batch == 0 || n == 0) return ABFT_OK;  // no element: not looked at
  const int es = es_of(c);
  const int64_t st[3] = {t->batch_stride, t->token_stride, t->head_stride};
  const int ext[3] = {c->batch, n, nh};
  if (!t->data || reinterpret_cast<uintptr_t>(t->data) % 16) return ABFT_ERR_INVALID;
  for (int k = 0; k < 3; ++k) {
    if (ext[k] == 1) continue;                  // the stride is not used
    if (st[k] < 0 || st[k] > MAX_EXTENT / es / ext[k] || (st[k] * es) % 16) return ABFT_ERR_INVALID;
  }
  if (out) {  // no element is written twice: from the smallest stride up, each passes the last
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return st[x] < st[y]; });
    int64_t extent = c->head_dim;
    for (int k : order) {
      if (ext[k] == 1) continue;
      if (st[k] < extent) return ABFT_ERR_INVALID;
      extent = st[k] * ext[k];
    }
  }
  if (n > 1 && st[1] * es > MAX_TOKEN_BYTES) return ABFT_ERR_UNSUPPORTED;
  r->p = static_cast<char*>(const_cast<void*>(t->data));
  r->b = c->batch > 1 ? st[0] * es : 0;
  r->t = n > 1 ? uint32_t(st[1] * es) : 0;
  r->h = nh > 1 ? st[2] * es : 0;
  return ABFT_OK;
}

// Whether a launch is in HIP's range (fewer than 2^32 threads). Only whole grids
// come near it; what splits an axis fills the chip at most.
bool launchable(int64_t wgs, int threads) { return wgs * threads < (int64_t(1) << 32); }

// The memory of an operand that `take` accepted.
Area area(const attn_cross_config* c, const attn_cross_tensor* t, int n, int nh) {
  const int es = es_of(c);
  if (c->batch == 0 || n == 0) return Area{};
  Area a = Area::flat(t->data, size_t(c->head_dim) * es);
  a.dim(0, t->batch_stride, c->batch, es);
  a.dim(1, t->token_stride, n, es);
  a.dim(2, t->head_stride, nh, es);
  return a;
}

// Whether one of the first n_out areas, which are written, shares memory with
// another area.
bool written_overlap(const Area* a, int n_out, int n) {
  for (int i = 0; i < n_out; ++i)
    for (int k = i + 1; k < n; ++k)
      if (overlap(a[i], a[k])) return true;
  return false;
}

void common(const attn_cross_config* c, const float* bias, const int32_t* k_lens,
            const int32_t* q_start, CrossArgs* a) {
  a->B = c->batch;
  a->Sq = c->q_len;
  a->Sk = c->k_len;
  a->nh = c->heads;
  a->kvh = c->kv_heads;
  a->group = c->heads / c->kv_heads;
  a->causal = c->causal;
  a->scale = c->scale > 0.f ? c->scale : 1.f / std::sqrt(float(c->head_dim));
  a->k_lens = k_lens;
  a->q_start = q_start;
  a->bias.table = bias;
}

}  // namespace
}  // namespace abft

using namespace abft;

#define TRY(x)                      \
  do {                              \
    const int st_ = (x);            \
    if (st_ != ABFT_OK) return st_; \
  } while (0)
#define CK(x)                                       \
  do {                                              \
    if ((x) != hipSuccess) return ABFT_ERR_HIP;     \
  } while (0)

extern "C" {

int attn_rel_bucket(int64_t relative, int32_t buckets, int32_t max_distance,
                    int32_t bidirectional) {
  CrossBias b;
  if (buckets < 1 || !make_bias(buckets, max_distance, bidirectional, &b)) return ABFT_ERR_INVALID;
  int base = 0;
  int64_t n = relative < -CROSS_MAX_DISTANCE ? -CROSS_MAX_DISTANCE
                                             : (relative > CROSS_MAX_DISTANCE ? CROSS_MAX_DISTANCE
                                                                              : relative);
  if (b.bidirectional) {
    base = n > 0 ? b.side : 0;
    n = n < 0 ? -n : n;
  } else {
    n = n < 0 ? -n : 0;
  }
  if (n < b.exact) return base + int(n);
  int k = b.exact;
  for (int i = 1; i < b.side - b.exact; ++i) k += n >= b.border[i] ? 1 : 0;
  return base + k;
}

size_t attn_cross_workspace_bytes(const attn_cross_config* cfg) {
  CrossBias b;
  if (validate(cfg, &b) != ABFT_OK) return 0;
  const Space L = make_space(cfg, plan_of(cfg, b));
  return std::max(std::max(L.fwd, L.bwd), ALIGN);
}

int attn_cross_forward(const attn_cross_config* cfg, const attn_cross_tensor* Q,
                       const attn_cross_tensor* K, const attn_cross_tensor* V, const float* bias,
                       const int32_t* k_lens, const int32_t* q_start, const attn_cross_tensor* O,
                       float* lse, void* rest, void* workspace, size_t workspace_bytes,
                       void* stream) {
  CrossArgs a;
  TRY(validate(cfg, &a.bias));
  if ((cfg->buckets > 0) != (bias != nullptr)) return ABFT_ERR_INVALID;
  TRY(take(cfg, Q, cfg->q_len, cfg->heads, false, &a.q));
  TRY(take(cfg, K, cfg->k_len, cfg->kv_heads, false, &a.k));
  TRY(take(cfg, V, cfg->k_len, cfg->kv_heads, false, &a.v));
  TRY(take(cfg, O, cfg->q_len, cfg->heads, true, &a.o));
  const Space L = make_space(cfg, plan_of(cfg, a.bias));
  if (L.fwd && !workspace) return ABFT_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 || reinterpret_cast<uintptr_t>(rest) % 16)
    return ABFT_ERR_INVALID;
  if (workspace_bytes < L.fwd) return ABFT_ERR_WORKSPACE;
  if (cfg->batch == 0 || cfg->q_len == 0) return ABFT_OK;
  const size_t rows = size_t(cfg->batch) * cfg->heads * cfg->q_len;
  const Area mem[] = {area(cfg, O, cfg->q_len, cfg->heads),
                      Area::flat(lse, rows * 4),
                      Area::flat(cfg->dtype == ABFT_BF16 ? rest : nullptr, rows * cfg->head_dim * 2),
                      Area::flat(workspace, L.fwd),
                      area(cfg, Q, cfg->q_len, cfg->heads),
                      area(cfg, K, cfg->k_len, cfg->kv_heads),
                      area(cfg, V, cfg->k_len, cfg->kv_heads),
                      Area::flat(bias, size_t(cfg->buckets) * cfg->heads * 4),
                      Area::flat(k_lens, size_t(cfg->batch) * 4),
                      Area::flat(q_start, size_t(cfg->batch) * 4)};
  if (written_overlap(mem, 4, 10)) return ABFT_ERR_INVALID;
  const bool is_short = short_form(cfg, &a.splits);
  const int64_t shared = int64_t(cfg->q_len) * (cfg->heads / cfg->kv_heads);
  if (!launchable(is_short ? int64_t(cfg->batch) * cfg->kv_heads * ((shared + 31) / 32) * a.splits
                           : int64_t(cfg->batch) * cfg->heads * cross_tiles(cfg->q_len, 128), 256))
    return ABFT_ERR_UNSUPPORTED;
  TRY(check_device());
  common(cfg, bias, k_lens, q_start, &a);
  a.lse = lse;
  a.rest = static_cast<char*>(rest);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (is_short) {
    char* ws = static_cast<char*>(workspace);
    a.part_o = reinterpret_cast<float*>(ws + L.part_o);
    a.part_ml = reinterpret_cast<float*>(ws + L.part_ml);
    CK(launch_cross_short(a, cfg->dtype, cfg->head_dim, s));
  } else {
    CK(launch_cross_fwd(a, cfg->dtype, cfg->head_dim, s));
  }
  return ABFT_OK;
}

int attn_cross_backward(const attn_cross_config* cfg, const attn_cross_tensor* dO,
                        const attn_cross_tensor* Q, const attn_cross_tensor* K,
                        const attn_cross_tensor* V, const attn_cross_tensor* O, const float* lse,
                        const void* rest, const float* bias, const int32_t* k_lens,
                        const int32_t* q_start, const attn_cross_tensor* dQ, const attn_cross_tensor* dK,
                        const attn_cross_tensor* dV, float* dbias, void* workspace,
                        size_t workspace_bytes, void* stream) {
  CrossArgs a;
  TRY(validate(cfg, &a.bias));
  if ((cfg->buckets > 0) != (bias != nullptr)) return ABFT_ERR_INVALID;
  if ((cfg->buckets > 0) != (dbias != nullptr)) return ABFT_ERR_INVALID;
  TRY(take(cfg, dO, cfg->q_len, cfg->heads, false, &a.dout));
  TRY(take(cfg, Q, cfg->q_len, cfg->heads, false, &a.q));
  TRY(take(cfg, K, cfg->k_len, cfg->kv_heads, false, &a.k));
  TRY(take(cfg, V, cfg->k_len, cfg->kv_heads, false, &a.v));
  TRY(take(cfg, O, cfg->q_len, cfg->heads, false, &a.o));
  TRY(take(cfg, dQ, cfg->q_len, cfg->heads, true, &a.dq));
  TRY(take(cfg, dK, cfg->k_len, cfg->kv_heads, true, &a.dk));
  TRY(take(cfg, dV, cfg->k_len, cfg->kv_heads, true, &a.dv));
  const bool any_q = cfg->batch > 0 && cfg->q_len > 0, any_k = cfg->batch > 0 && cfg->k_len > 0;
  if (any_q && !lse) return ABFT_ERR_INVALID;
  const CrossPlan plan = plan_of(cfg, a.bias);
  const Space L = make_space(cfg, plan);
  if (L.bwd && !workspace) return ABFT_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 || reinterpret_cast<uintptr_t>(rest) % 16)
    return ABFT_ERR_INVALID;
  if (workspace_bytes < L.bwd) return ABFT_ERR_WORKSPACE;
  const size_t rows = size_t(cfg->batch) * cfg->heads * cfg->q_len;
  const size_t table = size_t(cfg->buckets) * cfg->heads * 4;
  const Area mem[] = {area(cfg, dQ, cfg->q_len, cfg->heads),
                      area(cfg, dK, cfg->k_len, cfg->kv_heads),
                      area(cfg, dV, cfg->k_len, cfg->kv_heads),
                      Area::flat(dbias, table),
                      Area::flat(workspace, L.bwd),
                      area(cfg, dO, cfg->q_len, cfg->heads),
                      area(cfg, Q, cfg->q_len, cfg->heads),
                      area(cfg, K, cfg->k_len, cfg->kv_heads),
                      area(cfg, V, cfg->k_len, cfg->kv_heads),
                      area(cfg, O, cfg->q_len, cfg->heads),
                      Area::flat(lse, rows * 4),
                      Area::flat(cfg->dtype == ABFT_BF16 ? rest : nullptr, rows * cfg->head_dim * 2),
                      Area::flat(bias, table),
                      Area::flat(k_lens, size_t(cfg->batch) * 4),
                      Area::flat(q_start, size_t(cfg->batch) * 4)};
  if (written_overlap(mem, 5, 15)) return ABFT_ERR_INVALID;
  if (!launchable(int64_t(cfg->batch) * cfg->heads * cross_tiles(cfg->q_len, 128), 256) ||
      !launchable(int64_t(cfg->batch) * cfg->kv_heads * cross_tiles(cfg->k_len, 32 * plan.kv_keys) *
                      plan.kv_parts, 64 * plan.kv_keys * plan.kv_split) ||
      !launchable(cfg->buckets ? cfg->heads : 0, 256))
    return ABFT_ERR_UNSUPPORTED;
  TRY(check_device());
  common(cfg, bias, k_lens, q_start, &a);
  a.lse = const_cast<float*>(lse);
  a.rest = static_cast<char*>(const_cast<void*>(rest));
  char* ws = static_cast<char*>(workspace);
  a.q_pad = cross_tiles(cfg->q_len, CROSS_QT) * CROSS_QT;
  a.nlse = reinterpret_cast<float*>(ws);
  a.ndelta = reinterpret_cast<float*>(ws + L.ndelta);
  a.norm = reinterpret_cast<float*>(ws + L.norm);
  a.dbias_part = reinterpret_cast<float*>(ws + L.dbias);
  a.dbias = dbias;
  a.q_parts = plan.q_parts;
  a.kv_parts = plan.kv_parts;
  a.part_sum = reinterpret_cast<float*>(ws + L.sum);
  a.part_dq = a.part_dk = reinterpret_cast<float*>(ws + L.part);
  a.part_dv = reinterpret_cast<float*>(ws + L.part2);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (any_q) CK(launch_cross_bwd_q(a, plan, cfg->dtype, cfg->head_dim, s));
  if (any_k)
    CK(launch_cross_bwd_kv(a, plan, cfg->dtype, cfg->head_dim, s));
  else if (cfg->buckets)
    CK(launch_cross_no_keys(a, s));
  return ABFT_OK;
}

}  // extern "C"
