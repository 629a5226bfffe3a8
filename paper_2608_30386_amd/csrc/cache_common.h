// Host-side checks shared by the paged cache's entry points.
#pragma once

#include <cstdint>

#include "dasc/cache.h"

namespace dasc {

inline bool aligned_to(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A cache whose rows are aligned to `align` bytes
inline int check_cache(const dasc_kv_cache* c, int align) {
  if (!c) return DASC_E_INVAL;
  if (c->dtype != DASC_DTYPE_BF16 && c->dtype != DASC_DTYPE_F16) return DASC_E_INVAL;
  if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535 || c->head_dim < 8 ||
      c->head_dim > 256 || c->head_dim % 8)
    return DASC_E_SHAPE;
  if (!c->k || !c->v || !aligned_to(c->k, align) || !aligned_to(c->v, align)) return DASC_E_INVAL;
  for (const int64_t s : {c->k_page, c->k_tok, c->k_head, c->v_page, c->v_tok, c->v_head})
    if (s < 0 || s % (align / 2)) return DASC_E_INVAL;
  return DASC_OK;
}

}  // namespace dasc
