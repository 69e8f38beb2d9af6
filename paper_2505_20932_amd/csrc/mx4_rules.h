// Which kernel takes a layer on microscaled 4-bit operands (mx4_linear.hip).  Host arithmetic on sizes only, no HIP: the
// launcher and a CPU test share it.
#pragma once

#include <stdint.h>

#include "fast_rules.h"

namespace cwac {

// Split-K kernel with 16 x 16 or 32 x 32 (channels x tokens) tiles; tiles of 128 x 128 and 256 x 256.
enum { kMx4Split16 = 1, kMx4Split32 = 2, kMx4Tile128 = 3, kMx4Tile256 = 4 };

inline int mx4_split_form(int64_t m, int n, int k) { return m <= 16 ? kMx4Split16 : kMx4Split32; }

inline int mx4_form(int64_t m, int n, int k) {
  if (m >= 256 && n >= 256 && tiles_of(m, n, 256, 256) >= 128) return kMx4Tile256;
  if (m >= 128 && n >= 128 && tiles_of(m, n, 128, 128) >= 96) return kMx4Tile128;
  return mx4_split_form(m, n, k);
}

}  // namespace cwac
