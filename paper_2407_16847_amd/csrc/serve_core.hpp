// serve_core.hpp -- where a token lies in the paged cache: shared by the device
// kernels and the host tests.
#pragma once

#include <stdint.h>

#include "acsr_core.hpp"

namespace splat {

// Page of position `pos` of sequence b, -1 where it has none: the position is
// negative or past the table, or the table names no page of the cache.
SPLAT_HD int32_t page_of(const int32_t* pages, int32_t b, int32_t max_pages, int32_t n_pages,
                         int32_t page_shift, int64_t pos) {
  if (pos < 0 || (pos >> page_shift) >= max_pages) return -1;
  const int32_t p = pages[(int64_t)b * max_pages + (pos >> page_shift)];
  return p >= 0 && p < n_pages ? p : -1;
}

// Row of head h, in rows of d features, of the token at `pos` in page p.
SPLAT_HD uint32_t cache_row(int32_t p, int32_t heads, int32_t h, int32_t page_shift, int64_t pos) {
  return (((uint32_t)p * (uint32_t)heads + (uint32_t)h) << page_shift) +
         (uint32_t)(pos & (((int64_t)1 << page_shift) - 1));
}

}  // namespace splat
