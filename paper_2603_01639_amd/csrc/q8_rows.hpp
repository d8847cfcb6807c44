// Which blocks of an 8-bit cache's rows a call touches, in plain integers: the
// kernels' and, in a host build, their test's.
#pragma once

#include <stdint.h>

namespace ltd {

// Blocks of sr rows that `rows` consecutive rows can touch, wherever they begin.
constexpr int append_units(int rows, int sr) { return (rows + sr - 2) / sr + 1; }

// First row of the unit-th block that rows [P, P + n) touch, or -1 where they
// touch fewer.  (In 64 bits: a launch has units for the largest n and some to
// fill its workgroups, whose rows pass 2^31 where P and n may reach 2^30.)
constexpr int append_block(int P, int n, int unit, int sr) {
  const int64_t r0 = (static_cast<int64_t>(P / sr) + unit) * sr;
  return n > 0 && r0 < static_cast<int64_t>(P) + n ? static_cast<int>(r0) : -1;
}

}  // namespace ltd
