// A cache of pages as the kernels see it: byte strides, and where a position of a sequence lies.
#pragma once

#include "sale_common.h"

namespace sale {

struct PageSide {
  uint8_t* base;
  long long head;            // bytes, as are
  uint32_t page, token;
};

struct CacheView {
  PageSide k, v;
  const float *k_scale, *v_scale;
  const int32_t *table, *lens;
  int n_pages, page_shift, width;      // a page holds 1 << page_shift tokens; entries per table row
};

// What sale.h promises about p (validate_tokens comes first), c and its strides; table and lens only where they are used.
int validate_cache(const sale_params_t* p, const sale_cache_t* c, bool tables);
CacheView cache_view(const sale_params_t* p, const sale_cache_t* c);

}  // namespace sale
