// Host-side check of the rows of an output that a strided call writes.
#pragma once

#include <cstdint>

namespace dasc {

// Whether n0 x n1 rows of `width` elements, s0 and s1 elements from one to the next, lie apart: within the
// rows of the shorter stride first, and those as a whole within the longer.
inline bool rows_apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t width) {
  if (s0 < 0 || s1 < 0) return false;
  if (n0 == 0 || n1 == 0) return true;
  if (n0 <= 1) return n1 <= 1 || s1 >= width;
  if (n1 <= 1) return s0 >= width;
  const int64_t lo = s0 < s1 ? s0 : s1, hi = s0 < s1 ? s1 : s0;
  const int64_t n = s0 < s1 ? n0 : n1;          // rows that lie `lo` apart
  return lo >= width && hi / n >= lo;           // hi >= n lo, without the product
}

}  // namespace dasc
