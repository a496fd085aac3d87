// Global 2-norm of many gradient tensors, and clipping by it.
//
// norm = sqrt(sum over all elements of g^2); the squares of fp32 values, INF
// and NaN apart, are formed and summed in 64 bits, so neither a gradient of
// 1e30 nor one of 1e-30 is lost. The tensors pass as kernel arguments (no
// copy to the device), cut into chunks that workgroups take in turn; each
// workgroup leaves one partial sum, and every reader sums the partials in the
// same order: the result does not depend on scheduling. Bound by reading the
// gradients (and, for clipping, by reading them again and writing them).
#include <algorithm>
#include <cmath>
#include <utility>
#include <vector>

#include "abft_device.hpp"
#include "abft_internal.hpp"

namespace abft {
namespace {

constexpr int GRAD_TENSORS = 112;     // per launch: the arguments stay below 4 KB
constexpr int GRAD_CHUNK = 16384;     // elements a workgroup takes at a time
constexpr int GRAD_WGS = 1024;        // workgroups a launch at most: four a CU
constexpr int NT = 256;

struct GradPartial {
  double sum;
  int64_t bad;
};

struct GradList {
  const void* g[GRAD_TENSORS];
  void* out[GRAD_TENSORS];
  int64_t n[GRAD_TENSORS];
  int32_t first[GRAD_TENSORS + 1];    // chunks before each tensor
  uint8_t bf16[GRAD_TENSORS];
  int32_t count;
};

// tensor of a chunk: the last one whose first chunk is not behind it (empty
// tensors hold none)
__device__ __forceinline__ int tensor_of(const GradList& L, int chunk) {
  int lo = 0, hi = L.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (L.first[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ void add_square(float x, double& s, int& bad) {
  s = fma(double(x), double(x), s);
  bad += is_finite(x) ? 0 : 1;
}

__device__ __forceinline__ double wg_sum(double v, double* sh) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ void sum_chunk(const T* g, int n, double& s, int& bad) {
  constexpr int V = 16 / int(sizeof(T));
  int at = 0;
  if (reinterpret_cast<uintptr_t>(g) % 16 == 0) {
    const int nv = n / V;
    const u32x4* p = reinterpret_cast<const u32x4*>(g);
    constexpr int U = 4;
    int i = threadIdx.x;
    for (; i + (U - 1) * NT < nv; i += U * NT) {
      u32x4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = p[i + u * NT];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 2) {
            add_square(__uint_as_float(x[u][e] << 16), s, bad);
            add_square(__uint_as_float(x[u][e] & 0xffff0000u), s, bad);
          } else {
            add_square(__uint_as_float(x[u][e]), s, bad);
          }
        }
    }
    for (; i < nv; i += NT) {
      const u32x4 x = p[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
          add_square(__uint_as_float(x[e] << 16), s, bad);
          add_square(__uint_as_float(x[e] & 0xffff0000u), s, bad);
        } else {
          add_square(__uint_as_float(x[e]), s, bad);
        }
      }
    }
    at = nv * V;
  }
  for (int i = at + threadIdx.x; i < n; i += NT) add_square(Storage<T>::load(g[i]), s, bad);
}

__global__ __launch_bounds__(NT) void grad_sum_kernel(GradList L, GradPartial* part) {
  __shared__ double sh[4];
  double s = 0.0;
  int bad = 0;
  const int chunks = L.first[L.count];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int t = tensor_of(L, c);
    const int64_t at = int64_t(c - L.first[t]) * GRAD_CHUNK;
    const int n = int(min(int64_t(GRAD_CHUNK), L.n[t] - at));
    if (L.bf16[t])
      sum_chunk(static_cast<const bf16_t*>(L.g[t]) + at, n, s, bad);
    else
      sum_chunk(static_cast<const float*>(L.g[t]) + at, n, s, bad);
  }
  const double total = wg_sum(s, sh);
  const double nbad = wg_sum(double(bad), sh);
  if (threadIdx.x == 0) part[blockIdx.x] = GradPartial{total, int64_t(nbad)};
}

// The statistics of all partial sums, the same in every workgroup.
// `ratio`: coef before its rounding to fp32.
__device__ __forceinline__ abft_grad_stats stats_of(const GradPartial* part, int n, double max_norm,
                                                    double* sh, double* ratio) {
  double s = 0.0, bad = 0.0;
  for (int i = threadIdx.x; i < n; i += NT) {
    s += part[i].sum;
    bad += double(part[i].bad);
  }
  s = wg_sum(s, sh);
  bad = wg_sum(bad, sh);
  const double norm = sqrt(s);
  abft_grad_stats r;
  r.norm = float(norm);
  *ratio = bad == 0.0 && norm > max_norm ? max_norm / norm : 1.0;
  r.coef = float(*ratio);
  r.nonfinite = int64_t(bad);
  return r;
}

__global__ __launch_bounds__(NT) void grad_stats_kernel(const GradPartial* part, int n,
                                                        abft_grad_stats* stats) {
  __shared__ double sh[4];
  double ratio;
  const abft_grad_stats r = stats_of(part, n, double(__builtin_inff()), sh, &ratio);
  if (threadIdx.x == 0) *stats = r;
}

// The factor max_norm / norm as f * 2^e: below 2^-100 fp32 would hold fewer of its
// bits (none below 2^-149), while its product with a gradient of 1e38 is an
// ordinary number.
struct Factor {
  float f;
  int e;
  __device__ __forceinline__ float operator()(float x) const { return ldexpf(x * f, e); }
};
struct Plain {
  float f;
  __device__ __forceinline__ float operator()(float x) const { return x * f; }
};

template <typename T, typename F>
__device__ __forceinline__ u32x4 scaled(u32x4 x, F f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2)
      x[e] = uint32_t(f2bf(f(__uint_as_float(x[e] << 16)))) |
             (uint32_t(f2bf(f(__uint_as_float(x[e] & 0xffff0000u)))) << 16);
    else
      x[e] = __float_as_uint(f(__uint_as_float(x[e])));
  }
  return x;
}

template <typename T, typename F>
__device__ __forceinline__ void scale_chunk(const T* g, T* o, int n, F f) {
  constexpr int V = 16 / int(sizeof(T));
  int at = 0;
  if ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(o)) % 16 == 0) {
    const int nv = n / V;
    const u32x4* p = reinterpret_cast<const u32x4*>(g);
    u32x4* q = reinterpret_cast<u32x4*>(o);
    constexpr int U = 4;
    int i = threadIdx.x;
    for (; i + (U - 1) * NT < nv; i += U * NT) {
      u32x4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = __builtin_nontemporal_load(p + i + u * NT);
#pragma unroll
      for (int u = 0; u < U; ++u)
        __builtin_nontemporal_store(scaled<T>(x[u], f), q + i + u * NT);
    }
    for (; i < nv; i += NT) q[i] = scaled<T>(p[i], f);
    at = nv * V;
  }
  for (int i = at + threadIdx.x; i < n; i += NT)
    o[i] = Storage<T>::store(f(Storage<T>::load(g[i])));
}

// Chunks are taken from the last on: the end of what the sums read is still in
// the cache. Both the last reading and the result go past it (12 attention
// layers of 768 in fp32, tensors not in any cache before: 75.6 -> 60.0 us; 3.8
// TB/s of gradients read once and written once, 5.7 counting both readings).
__global__ __launch_bounds__(NT) void grad_scale_kernel(GradList L, const GradPartial* part,
                                                        int n_part, double max_norm,
                                                        abft_grad_stats* stats) {
  __shared__ double sh[4];
  double ratio;
  const abft_grad_stats r = stats_of(part, n_part, max_norm, sh, &ratio);
  if (stats && blockIdx.x == 0 && threadIdx.x == 0) *stats = r;
  Factor small = {r.coef, 0};
  if (ratio > 0.0 && ratio < 0x1p-100) {
    small.e = ilogb(ratio) + 1;  // (f < 1: no overflow in front of the shift)
    small.f = float(ldexp(ratio, -small.e));
  }
  const int chunks = L.first[L.count];
  for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
    const int c = chunks - 1 - k;
    const int t = tensor_of(L, c);
    if (r.coef == 1.f && L.out[t] == L.g[t]) continue;
    const int64_t at = int64_t(c - L.first[t]) * GRAD_CHUNK;
    const int n = int(min(int64_t(GRAD_CHUNK), L.n[t] - at));
    auto by_type = [&](auto f) {
      if (L.bf16[t])
        scale_chunk(static_cast<const bf16_t*>(L.g[t]) + at, static_cast<bf16_t*>(L.out[t]) + at,
                    n, f);
      else
        scale_chunk(static_cast<const float*>(L.g[t]) + at, static_cast<float*>(L.out[t]) + at, n,
                    f);
    };
    if (small.e == 0)
      by_type(Plain{r.coef});
    else
      by_type(small);
  }
}

bool valid_list(const abft_grad* g, int32_t n, bool out) {
  if (n < 0 || (n > 0 && !g)) return false;
  int64_t chunks = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (g[i].numel < 0) return false;
    if (g[i].dtype != ABFT_BF16 && g[i].dtype != ABFT_FP32) return false;
    const uintptr_t es = g[i].dtype == ABFT_FP32 ? 4 : 2;
    if (g[i].numel == 0) continue;
    if (!g[i].grad || reinterpret_cast<uintptr_t>(g[i].grad) % es) return false;
    if (out && (!g[i].out || reinterpret_cast<uintptr_t>(g[i].out) % es)) return false;
    if (g[i].numel > (int64_t(1) << 40)) return false;
    chunks += (g[i].numel + GRAD_CHUNK - 1) / GRAD_CHUNK;
    if (chunks > (1 << 30)) return false;
  }
  return true;
}

// Whether an output shares memory with another output or another gradient (an
// element would be scaled twice, or read after it was written).
bool outputs_overlap(const abft_grad* g, int32_t n) {
  struct Range {
    uintptr_t begin, end;
    bool out;
    int32_t i;
  };
  std::vector<Range> v;
  v.reserve(2 * size_t(n));
  for (int32_t i = 0; i < n; ++i) {
    if (g[i].numel == 0) continue;
    const uintptr_t bytes = uintptr_t(g[i].numel) * (g[i].dtype == ABFT_FP32 ? 4 : 2);
    const uintptr_t in = reinterpret_cast<uintptr_t>(g[i].grad);
    const uintptr_t out = reinterpret_cast<uintptr_t>(g[i].out);
    v.push_back({out, out + bytes, true, i});
    if (in != out) v.push_back({in, in + bytes, false, i});
  }
  std::sort(v.begin(), v.end(), [](const Range& x, const Range& y) { return x.begin < y.begin; });
  // the ends furthest up among outputs and among gradients so far
  uintptr_t end_out = 0, end_in = 0;
  for (const Range& r : v) {
    if (r.begin < end_out || (r.out && r.begin < end_in)) return true;
    uintptr_t& end = r.out ? end_out : end_in;
    end = std::max(end, r.end);
  }
  return false;
}

int launches(int32_t n) { return n == 0 ? 1 : (n + GRAD_TENSORS - 1) / GRAD_TENSORS; }

// Tensors [at, at + GRAD_TENSORS) of the list; returns the workgroups of
// their launch.
int fill(GradList* L, const abft_grad* g, int32_t n, int32_t at) {
  L->count = std::min(n - at, GRAD_TENSORS);
  int64_t chunks = 0;
  for (int i = 0; i < L->count; ++i) {
    const abft_grad& x = g[at + i];
    L->g[i] = x.grad;
    L->out[i] = x.out;
    L->n[i] = x.numel;
    L->bf16[i] = x.dtype == ABFT_BF16;
    L->first[i] = int32_t(chunks);
    chunks += (x.numel + GRAD_CHUNK - 1) / GRAD_CHUNK;
  }
  L->first[L->count] = int32_t(chunks);
  return int(std::max<int64_t>(1, std::min<int64_t>(chunks, GRAD_WGS)));
}

}  // namespace
}  // namespace abft

using namespace abft;

extern "C" {

size_t clip_gradients_workspace_bytes(int32_t n) {
  return n < 0 ? 0 : size_t(launches(n)) * GRAD_WGS * sizeof(GradPartial);
}

static int run_grads(const abft_grad* grads, int32_t n, bool clip, double max_norm,
                     abft_grad_stats* stats, void* workspace, size_t workspace_bytes,
                     void* stream) {
  if (!valid_list(grads, n, clip) || !stats || !workspace) return ABFT_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(stats) % 8 || reinterpret_cast<uintptr_t>(workspace) % 16)
    return ABFT_ERR_INVALID;
  if (clip && !(max_norm >= 0.0)) return ABFT_ERR_INVALID;
  try {
    if (clip && outputs_overlap(grads, n)) return ABFT_ERR_INVALID;
  } catch (...) {  // out of host memory
    return ABFT_ERR_INVALID;
  }
  if (workspace_bytes < clip_gradients_workspace_bytes(n)) return ABFT_ERR_WORKSPACE;
  const int st = check_device();
  if (st != ABFT_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  GradPartial* part = static_cast<GradPartial*>(workspace);
  GradList L;
  int parts = 0;
  for (int k = 0; k < launches(n); ++k) {
    const int wgs = fill(&L, grads, n, k * GRAD_TENSORS);
    grad_sum_kernel<<<dim3(wgs), NT, 0, s>>>(L, part + parts);
    if (hipGetLastError() != hipSuccess) return ABFT_ERR_HIP;
    parts += wgs;
  }
  if (!clip) {
    grad_stats_kernel<<<dim3(1), NT, 0, s>>>(part, parts, stats);
    return hipGetLastError() == hipSuccess ? ABFT_OK : ABFT_ERR_HIP;
  }
  for (int k = launches(n) - 1; k >= 0; --k) {
    const int wgs = fill(&L, grads, n, k * GRAD_TENSORS);
    grad_scale_kernel<<<dim3(wgs), NT, 0, s>>>(L, part, parts, max_norm,
                                               k == 0 ? stats : nullptr);
    if (hipGetLastError() != hipSuccess) return ABFT_ERR_HIP;
  }
  return ABFT_OK;
}

int global_grad_norm(const abft_grad* grads, int32_t n, abft_grad_stats* stats, void* workspace,
                     size_t workspace_bytes, void* stream) {
  return run_grads(grads, n, false, 0.0, stats, workspace, workspace_bytes, stream);
}

int clip_gradients(const abft_grad* grads, int32_t n, double max_norm, abft_grad_stats* stats,
                   void* workspace, size_t workspace_bytes, void* stream) {
  return run_grads(grads, n, true, max_norm, stats, workspace, workspace_bytes, stream);
}

}  // extern "C"
