// Dropout with an optional residual, y = residual + dropout(x), and its backward
// (the same without a residual). Which elements stay follows from their position
// and the generator's key alone, so no mask is stored. A thread takes chunks of
// eight elements of a row, which share one call of the generator. Bound by memory.
#include <algorithm>

#include "rows.hpp"

namespace abft {
namespace {

constexpr int NT = 256;
constexpr int U = 2;  // chunks of a thread

template <typename T, bool RES>
__global__ __launch_bounds__(NT) void dropout_kernel(DropoutArgs a, int64_t tiles) {
  const uint64_t seed = a.drop.threshold ? a.drop.rng[0] : 0;
  const uint64_t offset = a.drop.threshold ? a.drop.rng[1] : 0;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const uint64_t first = uint64_t(tile) * (NT * U);
    const uint32_t row0 = uint32_t(first / a.chunks.d);
    const uint32_t in_row = uint32_t(first - uint64_t(row0) * a.chunks.d);
    Chunk<T> c[U], r[U];
    T* out[U];
    uint32_t row[U], chunk[U];
    int m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = in_row + u * NT + threadIdx.x;
      const uint32_t down = a.chunks.quotient(i);
      row[u] = row0 + down;
      chunk[u] = i - down * a.chunks.d;
      m[u] = row[u] < uint32_t(a.rows) ? a.cols - int(8 * chunk[u]) : 0;
      if (m[u] <= 0) continue;
      RowAt at;
      at.b = a.tokens.quotient(row[u]);
      at.t = row[u] - at.b * a.tokens.d;
      load_chunk(c[u], row_of<T>(a.x, at) + 8 * chunk[u], m[u]);
      if constexpr (RES) load_chunk(r[u], row_of<T>(a.res, at) + 8 * chunk[u], m[u]);
      out[u] = row_of<T>(a.y, at) + 8 * chunk[u];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (m[u] <= 0) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = c[u].get(e);
      if (a.drop.threshold) drop(v, a.drop, seed, offset, row[u], chunk[u]);
      if constexpr (RES) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = plain_add(r[u].get(e), v[e]);
      }
      c[u].set(v);
      store_chunk(c[u], out[u], m[u]);
    }
  }
}

template <typename T> hipError_t launch(const DropoutArgs& a, hipStream_t s) {
  const int64_t chunks = int64_t(a.rows) * a.chunks.d;
  const int64_t tiles = (chunks + NT * U - 1) / (NT * U);
  const int grid = int(std::min<int64_t>(tiles, 1 << 20));
  if (a.res.p)
    dropout_kernel<T, true><<<dim3(grid), NT, 0, s>>>(a, tiles);
  else
    dropout_kernel<T, false><<<dim3(grid), NT, 0, s>>>(a, tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s) {
  return dtype == ABFT_BF16 ? launch<bf16_t>(a, s) : launch<float>(a, s);
}

}  // namespace abft
