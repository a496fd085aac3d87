// Division of whole numbers below 2^31 by one that is known before the launch:
// a product and a shift (plain arithmetic, for host and device).
#pragma once

#include <stdint.h>

#include "philox.hpp"

namespace abft {

// With 2^(l - 1) < d <= 2^l and m = ceil(2^(31 + l) / d) < 2^32: m d is less than
// 2^l above 2^(31 + l), so for n < 2^31 the product n m lies by less than 2^(31 + l)
// / d above n 2^(31 + l) / d, which reaches no further whole quotient.
struct Divisor {
  uint32_t d = 1, m = 1u << 31, shift = 31;

  static Divisor of(uint32_t d) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < d) ++l;
    Divisor r;
    r.d = d;
    r.shift = 31 + l;
    r.m = uint32_t(((uint64_t(1) << r.shift) + d - 1) / d);
    return r;
  }
  ABFT_BOTH uint32_t quotient(uint32_t n) const { return uint32_t((uint64_t(n) * m) >> shift); }
};

}  // namespace abft
