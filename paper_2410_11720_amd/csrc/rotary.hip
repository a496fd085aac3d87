// Rotary positions: pair k of a head at position p is turned by p f_k,
//   (a, c) -> m (a cos - c sin, a sin + c cos),
// backward by -p f_k. A workgroup takes some tokens: their angles' cosines and
// sines go to LDS once, then all heads of the tokens pass through. An angle is
// formed in 64 bits and reduced to one turn there (position 2^20 at one radian a
// position has 3 bits left behind the point in 32); its functions in 32. Bound by
// memory.
#include <algorithm>

#include "rotary_internal.hpp"
#include "rows.hpp"

namespace abft {
namespace {

constexpr int NT = 256;
constexpr int LDS_PAIRS = 4096;  // of a workgroup's tokens

template <typename T> __device__ __forceinline__ T* head_at(const HeadTensor& x, uint32_t b,
                                                            int64_t t, uint32_t h) {
  return reinterpret_cast<T*>(x.p + int64_t(b) * x.b + t * x.t + int64_t(h) * x.h);
}

template <typename T>
__device__ __forceinline__ void turn_halves(const T* x, T* o, const float2* cs, int half, int k) {
  const int m = half - k;
  Chunk<T> a, c;
  load_chunk(a, x + k, m);
  load_chunk(c, x + half + k, m);
  float p[8], q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 f = e < m ? cs[k + e] : make_float2(1.f, 0.f);
    p[e] = a.get(e) * f.x - c.get(e) * f.y;
    q[e] = a.get(e) * f.y + c.get(e) * f.x;
  }
  a.set(p);
  c.set(q);
  store_chunk(a, o + k, m);
  store_chunk(c, o + half + k, m);
}

template <typename T>
__device__ __forceinline__ void turn_neighbours(const T* x, T* o, const float2* cs, int half, int k) {
  const int m = 2 * (half - k);
  Chunk<T> a;
  load_chunk(a, x + 2 * k, m);
  float p[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = 2 * e < m ? cs[k + e] : make_float2(1.f, 0.f);
    p[2 * e] = a.get(2 * e) * f.x - a.get(2 * e + 1) * f.y;
    p[2 * e + 1] = a.get(2 * e) * f.y + a.get(2 * e + 1) * f.x;
  }
  a.set(p);
  store_chunk(a, o + 2 * k, m);
}

template <typename T>
__global__ __launch_bounds__(NT) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 cs[LDS_PAIRS];
  const int tiles = (a.n_tokens + a.tile - 1) / a.tile;
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int first = tile * a.tile, n = min(a.tile, a.n_tokens - first);
    __syncthreads();  // (the tile before has been read)
    for (int i = threadIdx.x; i < n * a.half; i += NT) {
      const int tok = i / a.half, k = i - tok * a.half;
      const uint32_t b = a.tokens.quotient(first + tok);
      const int64_t at = int64_t(a.start ? a.start[b] : 0) + (first + tok - int(b * a.tokens.d));
      double turns = double(at) * a.freqs[k] * 0.15915494309189533577;  // 1 / (2 pi)
      turns -= rint(turns);
      float s, c;
      sincospif(2.f * float(turns), &s, &c);
      cs[i] = make_float2(c * a.magnitude, s * a.magnitude * a.sign);
    }
    __syncthreads();
    const int items = n * int(a.slots.d * a.parts.d);
    for (int i = threadIdx.x; i < items; i += NT) {
      const uint32_t head = a.parts.quotient(i), part = i - head * a.parts.d;
      const uint32_t tok = a.slots.quotient(head);
      uint32_t slot = head - tok * a.slots.d;
      const uint32_t b = a.tokens.quotient(first + tok);
      const uint32_t t = first + tok - b * a.tokens.d;
      int which = 0;
      if (slot >= uint32_t(a.heads[0])) {
        slot -= a.heads[0];
        which = 1;
        if (slot >= uint32_t(a.heads[1])) {
          slot -= a.heads[1];
          which = 2;
        }
      }
      int64_t to = t;
      if (a.append && which > 0) {
        to += a.start ? a.start[b] : 0;
        if (to < 0 || to >= a.capacity) continue;
      }
      const HeadTensor& src = which == 0 ? a.in[0] : which == 1 ? a.in[1] : a.in[2];
      const HeadTensor& dst = which == 0 ? a.out[0] : which == 1 ? a.out[1] : a.out[2];
      const T* x = head_at<T>(src, b, t, slot);
      T* o = head_at<T>(dst, b, to, slot);
      const float2* f = cs + tok * a.half;
      if (which < 2 && part < uint32_t(a.turned)) {
        if (a.interleaved)
          turn_neighbours(x, o, f, a.half, 4 * part);
        else
          turn_halves(x, o, f, a.half, 8 * part);
        continue;
      }
      // dims that stay as they are: behind the turned ones, or all of a value's
      const int p0 = which < 2 ? 2 * a.half + 8 * (part - a.turned) : 8 * part;
      const int step = which < 2 ? a.head_dim : 8 * a.parts.d;
      for (int p = p0; p < a.head_dim; p += step) {
        Chunk<T> c;
        load_chunk(c, x + p, a.head_dim - p);
        store_chunk(c, o + p, a.head_dim - p);
      }
    }
  }
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int dtype, hipStream_t s) {
  a.turned = a.interleaved ? (a.half + 3) / 4 : (a.half + 7) / 8;
  const int parts = a.turned + (a.head_dim - 2 * a.half + 7) / 8;
  const int slots = a.heads[0] + a.heads[1] + a.heads[2];
  a.parts = Divisor::of(parts);
  a.slots = Divisor::of(slots);
  // tokens of a workgroup: four items a thread, but no fewer than 1024 workgroups
  const int64_t items = int64_t(parts) * slots;
  int64_t tile = std::max<int64_t>(1, 4 * NT / items);
  tile = std::min<int64_t>(tile, std::max(1, a.n_tokens / 1024));
  a.tile = int(std::min<int64_t>(tile, LDS_PAIRS / std::max(1, a.half)));
  const int tiles = (a.n_tokens + a.tile - 1) / a.tile;
  const int grid = std::min(tiles, 1 << 20);
  if (dtype == ABFT_BF16)
    rotary_kernel<bf16_t><<<dim3(grid), NT, 0, s>>>(a);
  else
    rotary_kernel<float><<<dim3(grid), NT, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace abft
