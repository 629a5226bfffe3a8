// Host-side helpers shared by the device entry points: shape validation and
// HIP launch-status mapping.  Nothing here runs on the GPU.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dasc.h"

namespace dasc {

inline bool valid_shape(const dasc_shape* s) {
  if (!s) return false;
  if (s->arch != DASC_ARCH_KDA && s->arch != DASC_ARCH_GDN) return false;
  if (s->n_layers <= 0 || s->n_heads <= 0 || s->n_qk_heads <= 0 || s->dk <= 0 || s->dv <= 0)
    return false;
  if (s->n_heads % s->n_qk_heads != 0) return false;
  const int64_t rows = int64_t(s->n_layers) * s->n_heads * s->dk;
  return rows < (int64_t(1) << 31);
}

inline int64_t rows_per_state(const dasc_shape* s) {
  return int64_t(s->n_layers) * s->n_heads * s->dk;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

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

// Map the launch status of the kernel just enqueued to a DASC status code.
inline int launch_status() {
  return hipGetLastError() == hipSuccess ? DASC_OK : DASC_E_HIP;
}

}  // namespace dasc
