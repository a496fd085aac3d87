// Whether two strided areas of memory share a byte (host only).
#pragma once

#include <stdint.h>

#include <algorithm>

namespace abft {

// Rows of `row` bytes, up to three dimensions of them with strides in bytes.
struct Area {
  uintptr_t at = 0, end = 0;  // of all rows; end == at: empty
  int64_t row = 0;
  int64_t stride[3] = {0, 0, 0};
  int64_t last[3] = {0, 0, 0};  // index of the last entry of each dimension

  static Area flat(const void* p, size_t bytes) {
    Area a;
    a.at = reinterpret_cast<uintptr_t>(p);
    a.end = p ? a.at + bytes : a.at;
    a.row = int64_t(bytes);
    return a;
  }
  // (stride of s units; not looked at in a dimension of extent 1)
  void dim(int k, int64_t s, int64_t n, int64_t unit = 1) {
    if (n < 2 || s == 0) return;
    stride[k] = s * unit;
    last[k] = n - 1;
    end += uintptr_t(stride[k]) * uintptr_t(n - 1);
  }
};

// Two rows meet where -a.row < (a.at - b.at) + sum x_k s_k < b.row, x_k the index
// into a dimension of either area; a stride that both have counts once, its x_k
// the difference of the indexes. From the longest stride down only the few x_k that
// the shorter ones can still bring into that range are tried: views of one
// packed tensor are told apart in some steps, whatever their size. An unusual
// pair that takes more than `budget` steps counts as apart.
struct Meeting {
  int64_t s[6], lo[6], hi[6], least[7], most[7];  // least, most: of the sum from k on
  int64_t below, above;
  int n = 0, budget = 4096;

  bool find(int k, int64_t d) {
    if (k == n) return d > below && d < above;
    // below < d + x s + rest < above for some rest in [least, most]
    const auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0 ? 1 : 0); };
    const int64_t from = std::max(lo[k], floor_div(below - d - most[k + 1], s[k]) + 1);
    const int64_t to = std::min(hi[k], -floor_div(-(above - d - least[k + 1]), s[k]) - 1);
    for (int64_t x = from; x <= to; ++x) {
      if (--budget < 0) return false;
      if (find(k + 1, d + x * s[k])) return true;
    }
    return false;
  }
};

inline bool overlap(const Area& a, const Area& b) {
  if (a.end == a.at || b.end == b.at || a.end <= b.at || b.end <= a.at) return false;
  Meeting m;
  auto put = [&](int64_t s, int64_t lo, int64_t hi) {
    for (int k = 0; k < m.n; ++k)
      if (m.s[k] == s) {
        m.lo[k] += lo;
        m.hi[k] += hi;
        return;
      }
    int k = m.n++;
    for (; k > 0 && m.s[k - 1] < s; --k) {
      m.s[k] = m.s[k - 1];
      m.lo[k] = m.lo[k - 1];
      m.hi[k] = m.hi[k - 1];
    }
    m.s[k] = s;
    m.lo[k] = lo;
    m.hi[k] = hi;
  };
  for (int k = 0; k < 3; ++k) {
    if (a.last[k]) put(a.stride[k], 0, a.last[k]);
    if (b.last[k]) put(b.stride[k], -b.last[k], 0);
  }
  m.least[m.n] = m.most[m.n] = 0;
  for (int k = m.n - 1; k >= 0; --k) {
    m.least[k] = m.least[k + 1] + m.lo[k] * m.s[k];
    m.most[k] = m.most[k + 1] + m.hi[k] * m.s[k];
  }
  m.below = -a.row;
  m.above = b.row;
  return m.find(0, int64_t(a.at - b.at));
}

}  // namespace abft
