// Rotary positions: pair k of a head at position p is turned by p f_k,
//   (a, c) -> m (a cos - c sin, a sin + c cos),
// backward by -p f_k. A wave, or 32 or 16 lanes of one, takes a token, or some heads of
// one: it forms the angles' cosines and sines once, into its own part of LDS, then its
// lanes take 16 dims of a head at a time. An angle is formed in 64 bits and reduced to
// one turn there (position 2^20 at one radian a position has 3 bits left behind the
// point in 32); its functions in 32. Bound by memory (4 x 2048 tokens, 40 heads on 8 of
// 128 dims in bf16: 45 us, 4.5 TB/s; in fp32 101 us, 4.0 TB/s).
#include <algorithm>

#include "rotary_internal.hpp"
#include "rows.hpp"

namespace abft {
namespace {

constexpr int NT = 256;
constexpr int MAX_PAIRS = 256;  // of a head

// Item: two chunks of a head, m[0] and m[1] of their elements in it.
template <typename T> struct Item {
  Chunk<T> c[2];
  T* out[2];
  int m[2];
  int pair;     // of the first element; below 0: copied
  bool store;
};

// L lanes a token, U items of a lane in flight. FULL: every chunk is whole.
template <typename T, int L, int U, bool INTER, bool FULL>
__global__ __launch_bounds__(NT) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 angles[NT / L][MAX_PAIRS * L / 64];
  const int lane = threadIdx.x % L;
  int group = threadIdx.x / L;
  if constexpr (L == 64) group = __builtin_amdgcn_readfirstlane(group);
  float2* cs = angles[group];
  const int jobs = a.n_tokens * int(a.waves.d);
  for (int64_t job = int64_t(blockIdx.x) * (NT / L) + group; job < jobs;
       job += int64_t(gridDim.x) * (NT / L)) {
    const uint32_t n = a.waves.quotient(uint32_t(job));
    const uint32_t b = a.tokens.quotient(n), t = n - b * a.tokens.d;
    const int first = int(uint32_t(job) - n * a.waves.d) * a.per;
    const int end = min(first + a.per, a.items);
    const int64_t pos = int64_t(a.start ? a.start[b] : 0) + t;
    const int64_t row = a.append ? pos : t;   // of keys and values
    const bool there = !a.append || (pos >= 0 && pos < a.capacity);
    auto at = [&](const HeadTensor& x, int64_t r) { return x.p + int64_t(b) * x.b + r * x.t; };
    const char *in0 = at(a.in[0], t), *in1 = at(a.in[1], t), *in2 = at(a.in[2], t);
    char *out0 = at(a.out[0], t), *out1 = at(a.out[1], row), *out2 = at(a.out[2], row);
    for (int k = lane; k < a.half; k += L) {
      double turns = double(pos) * a.freqs[k] * 0.15915494309189533577;  // 1 / (2 pi)
      turns -= rint(turns);
      float s, c;
      sincospif(2.f * float(turns), &s, &c);
      cs[k] = make_float2(c * a.magnitude, s * a.magnitude * a.sign);
    }
    // (a wave's LDS accesses keep their order)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    int i = first + lane;
    int head = a.parts.quotient(i), part = i - head * int(a.parts.d);
    while (i - lane < end) {
      Item<T> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        // (behind the last item: a first one again, not stored)
        const bool ok = i < end;
        const int h = ok ? head : 0, p = ok ? part : 0;
        const int which = h < a.heads[0] ? 0 : h < a.heads[0] + a.heads[1] ? 1 : 2;
        const int64_t slot = h - (which > 0 ? a.heads[0] : 0) - (which > 1 ? a.heads[1] : 0);
        const int64_t hs = which == 0 ? a.in[0].h : which == 1 ? a.in[1].h : a.in[2].h;
        const int64_t ho = which == 0 ? a.out[0].h : which == 1 ? a.out[1].h : a.out[2].h;
        const T* src = reinterpret_cast<const T*>((which == 0 ? in0 : which == 1 ? in1 : in2) +
                                                  slot * hs);
        T* dst = reinterpret_cast<T*>((which == 0 ? out0 : which == 1 ? out1 : out2) + slot * ho);
        const bool turn = which < 2 && p < a.turned;
        int e0, e1;
        if (turn) {
          x[u].pair = 8 * p;
          e0 = INTER ? 16 * p : 8 * p;
          e1 = INTER ? 16 * p + 8 : a.half + 8 * p;
          x[u].m[0] = INTER ? 2 * a.half - e0 : a.half - 8 * p;
          x[u].m[1] = INTER ? 2 * a.half - e1 : a.half - 8 * p;
        } else {
          x[u].pair = -1;
          e0 = 16 * p + (which < 2 ? 2 * a.half - 16 * a.turned : 0);
          e1 = e0 + 8;
          x[u].m[0] = a.head_dim - e0;
          x[u].m[1] = a.head_dim - e1;
        }
        x[u].out[0] = dst + e0;
        x[u].out[1] = dst + e1;
        x[u].store = ok && (which == 0 || there);
        if constexpr (FULL) {
          x[u].c[0].load(src + e0);
          x[u].c[1].load(src + e1);
        } else {
          load_chunk(x[u].c[0], src + e0, x[u].m[0]);
          load_chunk(x[u].c[1], src + e1, x[u].m[1]);
        }
        i += L;
        head += a.dq;
        part += a.dr;
        if (part >= int(a.parts.d)) {
          part -= a.parts.d;
          ++head;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (x[u].pair >= 0) {
          float p[8], q[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int k = x[u].pair + e;
            const float2 f = FULL ? cs[k] : cs[min(k, a.half - 1)];
            // elements of pair e: of both chunks, or neighbours in one
            Chunk<T>&ca = x[u].c[INTER ? e / 4 : 0], &cc = x[u].c[INTER ? e / 4 : 1];
            const int ia = INTER ? 2 * e % 8 : e, ic = INTER ? 2 * e % 8 + 1 : e;
            const float va = ca.get(ia), vc = cc.get(ic);
            p[e] = va * f.x - vc * f.y;
            q[e] = va * f.y + vc * f.x;
          }
          if constexpr (INTER) {
            const float lo[8] = {p[0], q[0], p[1], q[1], p[2], q[2], p[3], q[3]};
            const float hi[8] = {p[4], q[4], p[5], q[5], p[6], q[6], p[7], q[7]};
            x[u].c[0].set(lo);
            x[u].c[1].set(hi);
          } else {
            x[u].c[0].set(p);
            x[u].c[1].set(q);
          }
        }
        if (!x[u].store) continue;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if constexpr (FULL)
            x[u].c[k].store(x[u].out[k]);
          else
            store_chunk(x[u].c[k], x[u].out[k], x[u].m[k]);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T, int L, int U> hipError_t launch(RotaryArgs a, bool full, hipStream_t s) {
  a.dq = L / int(a.parts.d);
  a.dr = L % int(a.parts.d);
  // few tokens: several groups share one, down to an item a lane, up to 16 waves a CU (calls
  // one after another in bf16, 40 heads of 128 dims: 1024 tokens with 4 waves a CU 7.6, 16
  // 6.3, 64 6.7 us, 512 tokens 5.6, 5.1, 5.1; 24 heads of 64, 8192 tokens 13.1, 13.1, 16.2)
  const int steps = (a.items + L - 1) / L, few = 4096 * (64 / L);
  const int waves = std::max(1, std::min(steps, few / std::min(few, a.n_tokens)));
  a.per = L * ((steps + waves - 1) / waves);
  a.waves = Divisor::of((a.items + a.per - 1) / a.per);
  const int64_t jobs = int64_t(a.n_tokens) * a.waves.d;
  const dim3 grid(int(std::min<int64_t>((jobs + NT / L - 1) / (NT / L), 1 << 20)));
  auto* kernel = a.interleaved ? full ? rotary_kernel<T, L, U, true, true> : rotary_kernel<T, L, U, true, false>
                 : full        ? rotary_kernel<T, L, U, false, true>
                               : rotary_kernel<T, L, U, false, false>;
  return start(kernel, grid, NT, 0, s, a);
}

// Two items of a lane at once where there are more than lanes (calls one after another:
// 8192 tokens of 48 heads of 128 dims, half turned, 44.6 us, one at a time 46.3, 24 heads of
// 64 13.1 and 14.2; few tokens lose, 512 of 40 heads 5.1 and 4.7).
// Lanes a token: as many as it has items for (57 x 1257 tokens, three heads and three
// key heads of 80 dims, 30 items: a pass of both directions with 64 lanes 120, with 32
// 63 us).
template <typename T> hipError_t launch(const RotaryArgs& a, bool full, hipStream_t s) {
  if (a.items > 64) return launch<T, 64, 2>(a, full, s);
  if (a.items > 32 || a.half > MAX_PAIRS / 2) return launch<T, 64, 1>(a, full, s);
  if (a.items > 16 || a.half > MAX_PAIRS / 4) return launch<T, 32, 1>(a, full, s);
  return launch<T, 16, 1>(a, full, s);
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int dtype, hipStream_t s) {
  a.turned = (a.half + 7) / 8;
  const int copied = a.head_dim - 2 * a.half;
  const int parts = a.turned + (copied + 15) / 16;
  a.parts = Divisor::of(parts);
  a.items = parts * (a.heads[0] + a.heads[1] + a.heads[2]);
  const bool full = a.half % 8 == 0 && copied % 16 == 0;
  return dtype == ABFT_BF16 ? launch<bf16_t>(a, full, s) : launch<float>(a, full, s);
}

}  // namespace abft
