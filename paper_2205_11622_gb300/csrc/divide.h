// Division by a number that a whole launch shares (a page size, a group of
// heads): one multiplication and a shift.  Also compiled for the host.
#pragma once

#include <cstdint>

#include "range.h"

namespace slnr {

// Quotients of n in [0, 2^31) by a divisor d in [1, 2^31): with l = ceil(log2 d)
// and m = ceil(2^(31+l) / d), m < 2^32, and n m / 2^(31+l) exceeds n / d by less
// than n / (2^31 d), which never carries past the next whole number.
struct Divisor {
  uint32_t m;
  int shift;
  int d;
  SLNR_HD int div(int n) const { return (int)(((uint64_t)(uint32_t)n * m) >> shift); }
};

inline Divisor divisor(int d) {
  int l = 0;
  while ((int64_t(1) << l) < d) ++l;
  const uint64_t p = uint64_t(1) << (31 + l);
  return Divisor{(uint32_t)((p + d - 1) / d), 31 + l, d};
}

}  // namespace slnr
