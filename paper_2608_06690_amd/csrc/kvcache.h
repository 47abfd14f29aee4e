// Places in the paged cache, shared by its writer, its reader and the attention over it.
#pragma once
#include "pmpe_internal.h"

namespace pmpe {

// The tag that request r's pages have to carry (0 deny, 1 allow).
__device__ __forceinline__ uint32_t request_tag(const CacheArgs& c, int r) {
  return c.words && c.words[r] == PMPE_POLICY_ALLOW ? PMPE_POLICY_ALLOW : PMPE_POLICY_DENY;
}
// Page of column `col` of request r's table, or -1 with its bit in `bad` where the request may not use it.
__device__ __forceinline__ int page_at(const CacheArgs& c, int r, int64_t col, uint32_t want, uint32_t& bad) {
  if (col < 0 || col >= c.max_pages) {
    bad |= PMPE_DEV_CACHE_RANGE;
    return -1;
  }
  const int page = c.table[(size_t)r * c.max_pages + col];
  if (page < 0 || page >= c.n_pages) {
    bad |= PMPE_DEV_CACHE_RANGE;
    return -1;
  }
  if (c.tag && c.tag[page] != want) {
    bad |= PMPE_DEV_CACHE_REFUSED;
    return -1;
  }
  return page;
}
__device__ __forceinline__ void report(const CacheArgs& c, uint32_t bad) {
  if (bad && c.dev_status) atomicOr(c.dev_status, bad);
}

}  // namespace pmpe
