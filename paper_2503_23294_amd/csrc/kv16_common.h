// The paged 16-bit cache (cocktail_kv16_*): pages of [num_kv_heads][page_size][head_dim] in fp16 or bf16, a pool for K and one for V.
#pragma once
#include "paged_batch.h"

namespace cocktail {

int check_kv16_cache(const cocktail_kv16_cache* c);
// Rows [total][heads] of the cache's dtype.
int check_kv16_rows(const cocktail_kv16_cache* c, const void* x, const void* y, int64_t stride_t, int64_t stride_h, int64_t total, int heads);
// Bytes from the first of such rows to the end of the last (total > 0).
inline int64_t kv16_extent(const cocktail_kv16_cache* c, int64_t stride_t, int64_t stride_h, int64_t total, int heads) {
  return 2 * ((total - 1) * stride_t + (heads - 1) * stride_h + c->head_dim);
}
// Bytes of a pool (2^62 where 64 bits do not hold them).
inline int64_t kv16_pool_bytes(const cocktail_kv16_cache* c) {
  const double n = 2.0 * c->pages.num_pages * c->num_kv_heads * c->pages.page_size * c->head_dim;   // (exact up to 2^53)
  return n < 4.6e18 ? int64_t(n) : int64_t(1) << 62;
}
// The batch of a call, with K's pool; checks `total` against `starts`.
int check_kv16_batch(const cocktail_kv16_cache* c, int64_t total, const int32_t* starts, PagedBatch* a);

}  // namespace cocktail
