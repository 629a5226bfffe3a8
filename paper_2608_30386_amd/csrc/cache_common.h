// Host-side checks shared by the paged cache's entry points.
#pragma once

#include <cstdint>
#include <initializer_list>

#include "dasc/cache.h"

namespace dasc {

inline bool aligned_to(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The stride of a dimension of one element is never used, whatever it is: 0 stands for it.  (Negative ones are
// refused as everywhere.)
inline void drop_unused(int64_t n, std::initializer_list<int64_t*> strides) {
  if (n == 1)
    for (int64_t* s : strides)
      if (*s > 0) *s = 0;
}
inline void drop_unused(dasc_kv_cache& c) {
  drop_unused(c.n_pages, {&c.k_page, &c.v_page});
  drop_unused(c.page_size, {&c.k_tok, &c.v_tok});
  drop_unused(c.n_kv_heads, {&c.k_head, &c.v_head});
}

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
