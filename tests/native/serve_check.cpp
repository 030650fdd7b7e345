// serve_check.cpp -- the paged cache's address arithmetic on the host, built with
// the address and undefined-behaviour sanitizers: every position, good and bad,
// gives -1 or a row inside the cache, and good positions give distinct rows.
#include <cstdio>
#include <set>
#include <vector>

#include "../../paper_2407_16847_amd/csrc/serve_core.hpp"

using namespace splat;

int main() {
  const int32_t B = 3, heads = 5, max_pages = 4, n_pages = 12;
  for (int32_t shift : {0, 3, 16}) {
    std::vector<int32_t> table = {0, 5, 3, -1, 11, 12, 7, 1 << 30, 2, -2147483647 - 1, 9, 8};
    std::set<uint32_t> rows;
    const int64_t page = (int64_t)1 << shift, rows_all = n_pages * heads * page;
    for (int32_t b = 0; b < B; ++b) {
      std::vector<int64_t> at = {-9223372036854775807LL, -2147483648LL, -1, max_pages * page,
                                 2147483647LL, 4294967296LL};
      for (int64_t q = 0; q < max_pages; ++q)
        for (int64_t o : {(int64_t)0, page / 2, page - 1}) at.push_back(q * page + o);
      for (int64_t pos : std::set<int64_t>(at.begin(), at.end())) {
        const int32_t p = page_of(table.data(), b, max_pages, n_pages, shift, pos);
        const bool in = pos >= 0 && pos < max_pages * page;
        const int32_t want = in ? table[b * max_pages + pos / page] : -1;
        if (p != (want >= 0 && want < n_pages ? want : -1)) return 1;
        for (int32_t h = 0; p >= 0 && h < heads; ++h) {
          const uint32_t r = cache_row(p, heads, h, shift, pos);
          if ((int64_t)r >= rows_all || !rows.insert(r).second) return 2;
          if ((int64_t)r != ((int64_t)p * heads + h) * page + pos % page) return 3;
        }
      }
    }
  }
  // the largest cache: rows up to 2^32 - 1
  if (cache_row(65535, 1, 0, 16, 65535) != 0xffffffffu) return 4;
  std::puts("ok");
  return 0;
}
