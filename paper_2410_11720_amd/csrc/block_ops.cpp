// Host entry points of layer norm, dropout and rotary positions
// (include/attn_abft.h): checks and the kernels' arguments.
#include <algorithm>
#include <cmath>

#include "abft_internal.hpp"
#include "overlap.hpp"
#include "rotary_internal.hpp"
#include "rows.hpp"

namespace abft {
namespace {

constexpr int MAX_NORM_COLS = 16384;      // a row fits a workgroup's registers
constexpr int MAX_DROP_COLS = 65536;      // a chunk's number fits the counter's 13 bits
constexpr int64_t MAX_ROWS = 0x7ff00000;  // a row's number and one turn of a grid fit 31 bits
constexpr int MAX_SITE = 65536;
constexpr int MAX_HEAD_DIM = 512;
constexpr int MAX_HEADS = 65536;          // of queries, keys and values together
constexpr double MIN_EPS = 1e-30;         // squares below fp32's range stay far below it
constexpr double MAX_EPS = 1e37;          // variances of fp32's range and it have a sum there
constexpr int64_t MAX_EXTENT = int64_t(1) << 56;  // bytes between a dimension's ends

int es_of(int dtype) { return dtype == ABFT_FP32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == ABFT_BF16 || dtype == ABFT_FP32; }

// An operand of up to three strided dimensions over `row` contiguous elements.
struct Operand {
  Area area;
  const void* p = nullptr;
  int64_t st[3] = {0, 0, 0};  // bytes; 0 where the extent is below two
};

// `out`: no element may be written twice (from the smallest stride up, each passes
// the extent before).
int take(const void* p, const int64_t* st, const int* ext, int dims, int row, int es, bool out,
         Operand* r) {
  *r = Operand();
  for (int k = 0; k < dims; ++k)
    if (ext[k] == 0) return ABFT_OK;  // no element: not looked at
  if (!p || reinterpret_cast<uintptr_t>(p) % es) return ABFT_ERR_INVALID;
  int order[3] = {0, 1, 2};
  for (int k = 0; k < dims; ++k) {
    if (ext[k] == 1) continue;
    if (st[k] < 0 || st[k] > MAX_EXTENT / es / ext[k]) return ABFT_ERR_INVALID;
    r->st[k] = st[k] * es;
  }
  if (out) {
    std::sort(order, order + dims, [&](int x, int y) { return st[x] < st[y]; });
    int64_t extent = row;
    for (int i = 0; i < dims; ++i) {
      const int k = order[i];
      if (ext[k] == 1) continue;
      if (st[k] < extent) return ABFT_ERR_INVALID;
      extent = st[k] * ext[k];
    }
  }
  r->p = p;
  r->area = Area::flat(p, size_t(row) * es);
  for (int k = 0; k < dims; ++k) r->area.dim(k, st[k], ext[k], es);
  return ABFT_OK;
}

Operand vec(const void* p, size_t bytes) {
  Operand r;
  r.p = p;
  r.area = Area::flat(p, p ? bytes : 0);
  return r;
}

// The same elements in the same order.
bool same_place(const Operand& x, const Operand& y) {
  return x.p == y.p && x.area.row == y.area.row && x.area.end == y.area.end &&
         std::equal(x.st, x.st + 3, y.st);
}

// Whether one of the first n_out operands, which are written, shares memory with
// another one. An output may be one of the `in_place` operands behind them: each
// element of these is read by the thread that writes it, before it does.
bool written_overlap(const Operand* x, int n_out, int in_place, int n) {
  for (int i = 0; i < n_out; ++i)
    for (int k = i + 1; k < n; ++k) {
      if (k >= n_out && k < n_out + in_place && same_place(x[i], x[k])) continue;
      if (overlap(x[i].area, x[k].area)) return true;
    }
  return false;
}

int take_rows(int batch, int tokens, int cols, int dtype, const attn_rows* t, bool out, bool optional,
              Operand* r, RowTensor* to) {
  *r = Operand();
  if (!t || (!t->data && optional)) return optional ? ABFT_OK : ABFT_ERR_INVALID;
  const int64_t st[2] = {t->batch_stride, t->token_stride};
  const int ext[2] = {batch, tokens};
  const int e = take(t->data, st, ext, 2, cols, es_of(dtype), out, r);
  if (e != ABFT_OK) return e;
  to->p = static_cast<char*>(const_cast<void*>(t->data));
  to->b = r->st[0];
  to->t = r->st[1];
  return ABFT_OK;
}

int sizes_ok(int batch, int tokens, int cols, int most_cols) {
  if (batch < 0 || tokens < 0 || cols < 1) return ABFT_ERR_INVALID;
  if (cols > most_cols || int64_t(batch) * tokens > MAX_ROWS) return ABFT_ERR_UNSUPPORTED;
  return ABFT_OK;
}

int take_drop(double p, uint32_t site, const uint64_t* rng, DropArgs* d) {
  if (!(p >= 0.0 && p <= 1.0) || site >= MAX_SITE) return ABFT_ERR_INVALID;
  d->threshold = uint32_t(std::floor(65536.0 * p + 0.5));
  d->scale = d->threshold < 65536 ? float(65536.0 / (65536.0 - d->threshold)) : 0.f;
  d->last = uint32_t((uint64_t(d->threshold) << 16) - 1);
  d->site = site;
  d->rng = rng;
  if (d->threshold && (!rng || reinterpret_cast<uintptr_t>(rng) % 8)) return ABFT_ERR_INVALID;
  return ABFT_OK;
}

int valid_norm(const attn_norm_config* c) {
  if (!c || !dtype_ok(c->dtype) || !dtype_ok(c->weight_dtype)) return ABFT_ERR_INVALID;
  if (!(c->eps >= MIN_EPS && c->eps <= MAX_EPS)) return ABFT_ERR_INVALID;
  if (!(c->dropout >= 0.0 && c->dropout <= 1.0) || c->site >= MAX_SITE) return ABFT_ERR_INVALID;
  return sizes_ok(c->batch, c->tokens, c->cols, MAX_NORM_COLS);
}

size_t part_bytes(const attn_norm_config* c) {
  return size_t(norm_bwd_wgs(int64_t(c->batch) * c->tokens, c->cols)) * norm_part_stride(c->cols) * 4;
}

// Gains and offsets, lens, and what the kernels take from the config.
int common(const attn_norm_config* c, const void* weight, const void* bias, const int32_t* lens,
           NormArgs* a) {
  const int es = es_of(c->weight_dtype);
  if (reinterpret_cast<uintptr_t>(weight) % es || reinterpret_cast<uintptr_t>(bias) % es ||
      reinterpret_cast<uintptr_t>(lens) % 4)
    return ABFT_ERR_INVALID;
  a->weight = weight;
  a->bias = bias;
  a->weight_bf16 = c->weight_dtype == ABFT_BF16;
  a->lens = lens;
  a->rows = c->batch * c->tokens;
  a->cols = c->cols;
  a->tokens = Divisor::of(std::max(1, c->tokens));
  a->eps = c->eps;
  a->eps_scaled = c->eps * 0x1p-160;
  return ABFT_OK;
}

// How the rows of these tensors lie.
RowMode mode_of(const NormArgs& a, const Operand* rows, int n, int es) {
  if (a.rows == 0 || a.rows >= (1 << 28)) return ROWS_ANY;
  uintptr_t bits = uintptr_t(a.cols) * es;
  for (int i = 0; i < n; ++i) {
    if (!rows[i].p) continue;
    bits |= reinterpret_cast<uintptr_t>(rows[i].p) | uintptr_t(rows[i].st[0]) | uintptr_t(rows[i].st[1]);
    // (rows of less than a wave's width: 32-bit offsets from the tensor's start)
    const int64_t bytes = int64_t(rows[i].area.end - rows[i].area.at);
    if (a.cols <= NORM_LINE_COLS && bytes > 0x7fffff00) return ROWS_ANY;
  }
  if (a.cols % 8 == 0 && bits % 16 == 0) return ROWS_CHUNKS;
  return a.cols >= 8 && bits % 4 == 0 ? ROWS_WORDS : ROWS_ANY;
}

int valid_rotary(const attn_rotary_config* c) {
  if (!c || !dtype_ok(c->dtype)) return ABFT_ERR_INVALID;
  if (c->batch < 0 || c->tokens < 0 || c->heads < 0 || c->kv_heads < 0) return ABFT_ERR_INVALID;
  if (c->head_dim < 1 || c->rotary_dim < 0 || c->rotary_dim > c->head_dim || c->rotary_dim % 2)
    return ABFT_ERR_INVALID;
  if (c->interleaved != 0 && c->interleaved != 1) return ABFT_ERR_INVALID;
  if (!std::isfinite(c->magnitude)) return ABFT_ERR_INVALID;
  if (c->head_dim > MAX_HEAD_DIM || int64_t(c->heads) + 2 * int64_t(c->kv_heads) > MAX_HEADS ||
      int64_t(c->batch) * c->tokens > MAX_ROWS)
    return ABFT_ERR_UNSUPPORTED;
  return ABFT_OK;
}

int take_heads(const attn_rotary_config* c, const attn_cross_tensor* t, int tokens, int heads, bool out,
               Operand* r, HeadTensor* to) {
  *r = Operand();
  if (c->batch == 0 || tokens == 0 || heads == 0) return ABFT_OK;
  if (!t) return ABFT_ERR_INVALID;
  const int64_t st[3] = {t->batch_stride, t->token_stride, t->head_stride};
  const int ext[3] = {c->batch, tokens, heads};
  const int e = take(t->data, st, ext, 3, c->head_dim, es_of(c->dtype), out, r);
  if (e != ABFT_OK) return e;
  to->p = static_cast<char*>(const_cast<void*>(t->data));
  to->b = r->st[0];
  to->t = r->st[1];
  to->h = r->st[2];
  return ABFT_OK;
}

int rotary_common(const attn_rotary_config* c, const double* freqs, const int32_t* q_start,
                  RotaryArgs* a) {
  if (c->rotary_dim > 0 && !freqs) return ABFT_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(freqs) % 8 || reinterpret_cast<uintptr_t>(q_start) % 4)
    return ABFT_ERR_INVALID;
  a->heads[0] = c->heads;
  a->heads[1] = c->kv_heads;
  a->freqs = freqs;
  a->start = q_start;
  a->n_tokens = c->batch * c->tokens;
  a->tokens = Divisor::of(std::max(1, c->tokens));
  a->head_dim = c->head_dim;
  a->half = c->rotary_dim / 2;
  a->interleaved = c->interleaved;
  a->magnitude = c->magnitude > 0.f ? c->magnitude : 1.f;
  return ABFT_OK;
}

}  // namespace
}  // namespace abft

using namespace abft;

#define TRY(x)                      \
  do {                              \
    const int st_ = (x);            \
    if (st_ != ABFT_OK) return st_; \
  } while (0)
#define CK(x)                                   \
  do {                                          \
    if ((x) != hipSuccess) return ABFT_ERR_HIP; \
  } while (0)

extern "C" {

int attn_dropout_draw(uint64_t seed, uint64_t offset, uint32_t site, uint32_t row, uint32_t col) {
  if (site >= MAX_SITE || col >= MAX_DROP_COLS) return ABFT_ERR_INVALID;
  const Philox u = dropout_draws(seed, offset, site, row, col / 8);
  return int(u.w[col % 8 / 2] >> (col % 2 * 16) & 0xffffu);
}

int attn_dropout(const attn_dropout_config* cfg, const attn_rows* x, const attn_rows* residual,
                 const uint64_t* rng, const attn_rows* y, void* stream) {
  if (!cfg || !dtype_ok(cfg->dtype)) return ABFT_ERR_INVALID;
  TRY(sizes_ok(cfg->batch, cfg->tokens, cfg->cols, MAX_DROP_COLS));
  DropoutArgs a;
  TRY(take_drop(cfg->dropout, cfg->site, rng, &a.drop));
  Operand mem[4];
  const int B = cfg->batch, S = cfg->tokens, H = cfg->cols, dt = cfg->dtype;
  TRY(take_rows(B, S, H, dt, y, true, false, &mem[0], &a.y));
  TRY(take_rows(B, S, H, dt, x, false, false, &mem[1], &a.x));
  TRY(take_rows(B, S, H, dt, residual, false, true, &mem[2], &a.res));
  mem[3] = vec(rng, a.drop.threshold ? 16 : 0);
  if (written_overlap(mem, 1, 2, 4)) return ABFT_ERR_INVALID;
  a.rows = B * S;
  a.cols = H;
  if (a.rows == 0) return ABFT_OK;
  a.tokens = Divisor::of(S);
  a.chunks = Divisor::of((H + 7) / 8);
  a.flat = H % 8 == 0;
  for (int i = 0; i < 3; ++i) {
    if (!mem[i].p) continue;
    const int64_t row = int64_t(H) * es_of(dt);
    if (reinterpret_cast<uintptr_t>(mem[i].p) % 16 || (S > 1 && mem[i].st[1] != row) ||
        (B > 1 && mem[i].st[0] != row * S))
      a.flat = 0;
  }
  TRY(check_device());
  CK(launch_dropout(a, dt, static_cast<hipStream_t>(stream)));
  return ABFT_OK;
}

size_t attn_norm_workspace_bytes(const attn_norm_config* cfg) {
  return valid_norm(cfg) == ABFT_OK ? part_bytes(cfg) : 0;
}

int attn_norm_forward(const attn_norm_config* cfg, const attn_rows* x, const attn_rows* residual,
                      const void* weight, const void* bias, const int32_t* lens, const uint64_t* rng,
                      const attn_rows* h, const attn_rows* y, float* stats, void* stream) {
  TRY(valid_norm(cfg));
  NormArgs a;
  TRY(take_drop(cfg->dropout, cfg->site, rng, &a.drop));
  const bool sum = residual && residual->data, none = cfg->batch == 0 || cfg->tokens == 0;
  if (!none && !sum && (a.drop.threshold || (h && h->data))) return ABFT_ERR_INVALID;
  TRY(common(cfg, weight, bias, lens, &a));
  if (reinterpret_cast<uintptr_t>(stats) % 8) return ABFT_ERR_INVALID;
  const int B = cfg->batch, S = cfg->tokens, H = cfg->cols, dt = cfg->dtype;
  Operand mem[9];
  TRY(take_rows(B, S, H, dt, y, true, false, &mem[0], &a.y));
  TRY(take_rows(B, S, H, dt, h, true, true, &mem[1], &a.h));
  mem[2] = vec(stats, size_t(a.rows) * 8);
  TRY(take_rows(B, S, H, dt, x, false, false, &mem[3], &a.x));
  TRY(take_rows(B, S, H, dt, residual, false, true, &mem[4], &a.res));
  const size_t params = size_t(H) * es_of(cfg->weight_dtype);
  mem[5] = vec(weight, params);
  mem[6] = vec(bias, params);
  mem[7] = vec(lens, size_t(B) * 4);
  mem[8] = vec(rng, a.drop.threshold ? 16 : 0);
  if (written_overlap(mem, 3, 2, 9)) return ABFT_ERR_INVALID;
  if (a.rows == 0) return ABFT_OK;
  a.stats = reinterpret_cast<float2*>(stats);
  const Operand rows[] = {mem[0], mem[1], mem[3], mem[4]};
  a.mode = mode_of(a, rows, 4, es_of(dt));
  TRY(check_device());
  CK(launch_norm_fwd(a, dt, a.drop.threshold ? NORM_DROPOUT : sum ? NORM_RESIDUAL : NORM_ALONE,
                     static_cast<hipStream_t>(stream)));
  return ABFT_OK;
}

int attn_norm_backward(const attn_norm_config* cfg, const attn_rows* dy, const attn_rows* dh,
                       const attn_rows* h, const void* weight, const float* stats,
                       const int32_t* lens, const uint64_t* rng, const attn_rows* dx,
                       const attn_rows* dresidual, float* dweight, float* dbias, void* workspace,
                       size_t workspace_bytes, void* stream) {
  TRY(valid_norm(cfg));
  NormArgs a;
  TRY(take_drop(cfg->dropout, cfg->site, rng, &a.drop));
  TRY(common(cfg, weight, nullptr, lens, &a));
  const bool grads = dweight || dbias;
  if (reinterpret_cast<uintptr_t>(stats) % 8 || reinterpret_cast<uintptr_t>(workspace) % 16 ||
      reinterpret_cast<uintptr_t>(dweight) % 4 || reinterpret_cast<uintptr_t>(dbias) % 4)
    return ABFT_ERR_INVALID;
  if ((a.rows && !stats) || (grads && !workspace)) return ABFT_ERR_INVALID;
  const size_t part = grads ? part_bytes(cfg) : 0;
  if (workspace_bytes < part) return ABFT_ERR_WORKSPACE;
  const int B = cfg->batch, S = cfg->tokens, H = cfg->cols, dt = cfg->dtype;
  Operand mem[12];
  TRY(take_rows(B, S, H, dt, dx, true, true, &mem[0], &a.dx));
  TRY(take_rows(B, S, H, dt, dresidual, true, true, &mem[1], &a.dres));
  mem[2] = vec(dweight, size_t(H) * 4);
  mem[3] = vec(dbias, size_t(H) * 4);
  mem[4] = vec(workspace, part);
  TRY(take_rows(B, S, H, dt, dy, false, false, &mem[5], &a.dy));
  TRY(take_rows(B, S, H, dt, dh, false, true, &mem[6], &a.dh));
  TRY(take_rows(B, S, H, dt, h, false, false, &mem[7], &a.h));
  mem[8] = vec(weight, size_t(H) * es_of(cfg->weight_dtype));
  mem[9] = vec(stats, size_t(a.rows) * 8);
  mem[10] = vec(lens, size_t(B) * 4);
  mem[11] = vec(rng, a.drop.threshold ? 16 : 0);
  if (written_overlap(mem, 5, 3, 12)) return ABFT_ERR_INVALID;
  a.stats = reinterpret_cast<float2*>(const_cast<float*>(stats));
  a.dweight = dweight;
  a.dbias = dbias;
  a.part = static_cast<float*>(workspace);
  a.stride = norm_part_stride(H);
  if (a.rows == 0 && !grads) return ABFT_OK;
  const Operand rows[] = {mem[0], mem[1], mem[5], mem[6], mem[7]};
  a.mode = mode_of(a, rows, 5, es_of(dt));
  TRY(check_device());
  const bool sum = a.dres.p || a.dh.p;
  CK(launch_norm_bwd(a, dt, a.drop.threshold ? NORM_DROPOUT : sum ? NORM_RESIDUAL : NORM_ALONE,
                     static_cast<hipStream_t>(stream)));
  return ABFT_OK;
}

int attn_rotary_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor,
                            double original_len, double low_turns, double high_turns, double* freqs) {
  if (rotary_dim < 0 || rotary_dim % 2 || rotary_dim > MAX_HEAD_DIM || (rotary_dim && !freqs))
    return ABFT_ERR_INVALID;
  if (!(base > 0.0) || !std::isfinite(base)) return ABFT_ERR_INVALID;
  if (scaling < ABFT_ROTARY_PLAIN || scaling > ABFT_ROTARY_PARTS) return ABFT_ERR_INVALID;
  if (scaling != ABFT_ROTARY_PLAIN && (!(factor > 0.0) || !std::isfinite(factor)))
    return ABFT_ERR_INVALID;
  if (scaling == ABFT_ROTARY_PARTS &&
      (!(original_len > 0.0) || !std::isfinite(original_len) || !(low_turns >= 0.0) ||
       !(high_turns > low_turns) || !std::isfinite(high_turns)))
    return ABFT_ERR_INVALID;
  for (int k = 0; k < rotary_dim / 2; ++k) {
    double f = std::pow(base, -2.0 * k / rotary_dim);
    if (scaling == ABFT_ROTARY_LINEAR) f /= factor;
    if (scaling == ABFT_ROTARY_PARTS) {
      const double turns = original_len * f / (2.0 * M_PI);
      const double keep =
          std::min(1.0, std::max(0.0, (turns - low_turns) / (high_turns - low_turns)));
      f = f / factor * (1.0 - keep) + f * keep;
    }
    freqs[k] = f;
  }
  return ABFT_OK;
}

int attn_rotary(const attn_rotary_config* cfg, int32_t backward, const attn_cross_tensor* Q,
                const attn_cross_tensor* K, const double* freqs, const int32_t* q_start,
                const attn_cross_tensor* Q_out, const attn_cross_tensor* K_out, void* stream) {
  TRY(valid_rotary(cfg));
  if (backward != 0 && backward != 1) return ABFT_ERR_INVALID;
  RotaryArgs a;
  TRY(rotary_common(cfg, freqs, q_start, &a));
  a.sign = backward ? -1.f : 1.f;
  Operand mem[6];
  TRY(take_heads(cfg, Q_out, cfg->tokens, cfg->heads, true, &mem[0], &a.out[0]));
  TRY(take_heads(cfg, K_out, cfg->tokens, cfg->kv_heads, true, &mem[1], &a.out[1]));
  TRY(take_heads(cfg, Q, cfg->tokens, cfg->heads, false, &mem[2], &a.in[0]));
  TRY(take_heads(cfg, K, cfg->tokens, cfg->kv_heads, false, &mem[3], &a.in[1]));
  // in place: queries on queries, keys on keys
  const bool q_same = same_place(mem[0], mem[2]), k_same = same_place(mem[1], mem[3]);
  if ((!q_same && overlap(mem[0].area, mem[2].area)) || (!k_same && overlap(mem[1].area, mem[3].area)) ||
      overlap(mem[0].area, mem[3].area) || overlap(mem[1].area, mem[2].area))
    return ABFT_ERR_INVALID;
  mem[2] = vec(freqs, size_t(a.half) * 8);
  mem[3] = vec(q_start, size_t(cfg->batch) * 4);
  if (written_overlap(mem, 2, 0, 4)) return ABFT_ERR_INVALID;
  if (a.n_tokens == 0 || a.heads[0] + a.heads[1] == 0) return ABFT_OK;
  TRY(check_device());
  CK(launch_rotary(a, cfg->dtype, static_cast<hipStream_t>(stream)));
  return ABFT_OK;
}

int attn_rotary_append(const attn_rotary_config* cfg, const attn_cross_tensor* Q,
                       const attn_cross_tensor* K, const attn_cross_tensor* V, const double* freqs,
                       const int32_t* q_start, int32_t capacity, const attn_cross_tensor* Q_out,
                       const attn_cross_tensor* K_cache, const attn_cross_tensor* V_cache,
                       void* stream) {
  TRY(valid_rotary(cfg));
  if (capacity < 0) return ABFT_ERR_INVALID;
  RotaryArgs a;
  TRY(rotary_common(cfg, freqs, q_start, &a));
  a.heads[2] = cfg->kv_heads;
  a.append = 1;
  a.capacity = capacity;
  const int S = cfg->tokens, kvh = cfg->kv_heads;
  Operand mem[8];
  TRY(take_heads(cfg, Q_out, S, cfg->heads, true, &mem[0], &a.out[0]));
  TRY(take_heads(cfg, K_cache, capacity, kvh, true, &mem[1], &a.out[1]));
  TRY(take_heads(cfg, V_cache, capacity, kvh, true, &mem[2], &a.out[2]));
  TRY(take_heads(cfg, Q, S, cfg->heads, false, &mem[3], &a.in[0]));
  TRY(take_heads(cfg, K, S, kvh, false, &mem[4], &a.in[1]));
  TRY(take_heads(cfg, V, S, kvh, false, &mem[5], &a.in[2]));
  mem[6] = vec(freqs, size_t(a.half) * 8);
  mem[7] = vec(q_start, size_t(cfg->batch) * 4);
  // in place: queries on queries
  if (same_place(mem[0], mem[3])) mem[3] = Operand();
  if (written_overlap(mem, 3, 0, 8)) return ABFT_ERR_INVALID;
  if (a.n_tokens == 0 || cfg->heads + kvh == 0) return ABFT_OK;
  TRY(check_device());
  CK(launch_rotary(a, cfg->dtype, static_cast<hipStream_t>(stream)));
  return ABFT_OK;
}

}  // extern "C"
