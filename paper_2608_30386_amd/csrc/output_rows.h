// Host-side check of the rows of an output that a strided call writes.
#pragma once

#include <cstdint>

namespace dasc {

// Whether n0 x n1 rows of `width` elements, s0 and s1 elements from one to the next, lie apart: within the
// rows of the shorter stride first, and those as a whole, from the first one's start to the last one's end, within
// the longer.  (Rows of one kind that lie in the gaps of the other are not looked for.)
inline bool rows_apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t width) {
  if (s0 < 0 || s1 < 0) return false;
  if (n0 == 0 || n1 == 0) return true;
  if (n0 <= 1) return n1 <= 1 || s1 >= width;
  if (n1 <= 1) return s0 >= width;
  const int64_t lo = s0 < s1 ? s0 : s1, hi = s0 < s1 ? s1 : s0;
  const int64_t n = s0 < s1 ? n0 : n1;          // rows that lie `lo` apart
  return lo >= width && hi >= width && (hi - width) / (n - 1) >= lo;   // hi >= (n - 1) lo + width, without the product
}

// The same for n0 x n1 x n2 rows: in order of their strides, each kind as a whole within the next.
inline bool rows_apart3(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t width) {
  int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
  for (int i = 0; i < 3; ++i) {
    if (s[i] < 0) return false;
    if (n[i] == 0) return true;
  }
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (s[j] > s[j + 1]) {
        const int64_t ts = s[j], tn = n[j];
        s[j] = s[j + 1], n[j] = n[j + 1];
        s[j + 1] = ts, n[j + 1] = tn;
      }
  int64_t span = width;                         // that the rows so far take
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if (s[i] < span || s[i] > (INT64_MAX - span) / (n[i] - 1)) return false;
    span += s[i] * (n[i] - 1);
  }
  return true;
}

}  // namespace dasc
