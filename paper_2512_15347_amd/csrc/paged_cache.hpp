// The paged key/value cache of a token policy: what its kernels share.
#pragma once
#include "common.hpp"

namespace pg {

// status bits of pg_cache.status beside those of the selection (1, 2)
constexpr int CACHE_FULL = 4, CACHE_RANGE = 8;

// Checks the descriptor alone; `data`: the pools are needed, too.
pg_status check_cache(const pg_cache* c, bool data, const char* who);

// The descriptor as kernels take it.
struct CacheView {
  int32_t n_pages, heads, width, page_shift;
  int32_t* status;
};
inline CacheView view_of(const pg_cache* c) {
  return CacheView{c->n_pages, c->heads, c->width, __builtin_ctz((unsigned)c->page), c->status};
}
inline size_t cache_elt(const pg_cache* c) { return c->dtype == PG_CACHE_E4M3 ? 1 : 2; }
// bytes of one page of one layer, keys or values
inline size_t page_bytes(const pg_cache* c) { return (size_t)c->heads * c->page * c->head_dim * cache_elt(c); }

}  // namespace pg
