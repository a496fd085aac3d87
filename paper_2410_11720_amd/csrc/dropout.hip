// Dropout with an optional residual, y = residual + dropout(x), and its backward
// (the same without a residual). Which elements stay follows from their position
// and the generator's key alone, so no mask is stored. A thread takes chunks of
// eight elements of a row, which share one call of the generator. Bound by memory (8192
// x 16384 in bf16: 94 us, 5.7 TB/s; 8192 x 8192 in fp32: 122 us, 4.4 TB/s).
#include <algorithm>

#include "rows.hpp"

namespace abft {
namespace {

constexpr int NT = 256;
constexpr int U = 2;  // chunks of a thread, where rows have no gaps

template <typename T, bool RES>
__device__ __forceinline__ void apply(Chunk<T>& c, const Chunk<T>& r, const DropArgs& d, uint64_t seed,
                                      uint64_t offset, uint32_t row, uint32_t chunk) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c.get(e);
  if (d.threshold) drop(v, d, seed, offset, row, chunk);
  if constexpr (RES) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = plain_add(r.get(e), v[e]);
  }
  c.set(v);
}

// Tensors without gaps: a chunk's place is its number (calls one after another, with a
// residual in bf16: 8192 x 768 7.8 us, by rows 8.2; 4096 x 5120 24.6, by rows 25.8).
template <typename T, bool RES, bool PAST>
__global__ __launch_bounds__(NT) void dropout_flat(DropoutArgs a, int64_t chunks, int64_t tiles) {
  const uint64_t seed = a.drop.threshold ? a.drop.rng[0] : 0;
  const uint64_t offset = a.drop.threshold ? a.drop.rng[1] : 0;
  const T* x = reinterpret_cast<const T*>(a.x.p);
  const T* res = reinterpret_cast<const T*>(a.res.p);
  T* y = reinterpret_cast<T*>(a.y.p);
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const uint64_t first = uint64_t(tile) * (NT * U);
    const uint32_t row0 = uint32_t(first / a.chunks.d);
    const uint32_t in_row = uint32_t(first - uint64_t(row0) * a.chunks.d);
    Chunk<T> c[U], r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // (behind the last chunk: that one again, not stored)
      const int64_t i = min(int64_t(first) + u * NT + threadIdx.x, chunks - 1);
      c[u].load(x + 8 * i);
      if constexpr (RES) r[u].load(res + 8 * i);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t k = in_row + u * NT + threadIdx.x, down = a.chunks.quotient(k);
      apply<T, RES>(c[u], r[u], a.drop, seed, offset, row0 + down, k - down * a.chunks.d);
      const int64_t i = int64_t(first) + u * NT + threadIdx.x;
      if (i >= chunks) continue;
      if constexpr (PAST)
        c[u].store_past(y + 8 * i);
      else
        c[u].store(y + 8 * i);
    }
  }
}

// Any rows, a chunk a thread (8192 x 1001 with a residual in bf16: 11.7 us; two 13.1).
template <typename T, bool RES>
__global__ __launch_bounds__(NT) void dropout_rows(DropoutArgs a, int64_t tiles) {
  const uint64_t seed = a.drop.threshold ? a.drop.rng[0] : 0;
  const uint64_t offset = a.drop.threshold ? a.drop.rng[1] : 0;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const uint64_t first = uint64_t(tile) * NT;
    const uint32_t row0 = uint32_t(first / a.chunks.d);
    const uint32_t i = uint32_t(first - uint64_t(row0) * a.chunks.d) + threadIdx.x;
    const uint32_t down = a.chunks.quotient(i), row = row0 + down, chunk = i - down * a.chunks.d;
    if (row >= uint32_t(a.rows)) return;
    const int m = a.cols - int(8 * chunk);
    const RowAt at = row_at(a.tokens, row);
    Chunk<T> c, r;
    load_chunk(c, row_of<T>(a.x, at) + 8 * chunk, m);
    if constexpr (RES) load_chunk(r, row_of<T>(a.res, at) + 8 * chunk, m);
    apply<T, RES>(c, r, a.drop, seed, offset, row, chunk);
    store_chunk(c, row_of<T>(a.y, at) + 8 * chunk, m);
  }
}

// A result of this many bytes goes past the cache: what reads it next finds less than
// half of it there anyway (bf16, dropout alone, and with a pass that reads its
// result: 128 MiB 57 -> 49, 75 -> 71 us; 256 MiB 110 -> 94, 150 -> 133 us; below, a
// reader that takes it in parts loses more than this gains).
constexpr int64_t PAST_BYTES = int64_t(128) << 20;

template <typename T, bool RES> hipError_t launch(const DropoutArgs& a, hipStream_t s) {
  const int64_t chunks = int64_t(a.rows) * a.chunks.d;
  const int64_t per = a.flat ? NT * U : NT, tiles = (chunks + per - 1) / per;
  const dim3 grid(int(std::min<int64_t>(tiles, 1 << 20)));
  if (!a.flat) return start(dropout_rows<T, RES>, grid, NT, 0, s, a, tiles);
  const bool past = chunks * 8 * int64_t(sizeof(T)) >= PAST_BYTES;
  return start(past ? dropout_flat<T, RES, true> : dropout_flat<T, RES, false>, grid, NT, 0, s, a,
               chunks, tiles);
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s) {
  if (dtype == ABFT_BF16) return a.res.p ? launch<bf16_t, true>(a, s) : launch<bf16_t, false>(a, s);
  return a.res.p ? launch<float, true>(a, s) : launch<float, false>(a, s);
}

}  // namespace abft
