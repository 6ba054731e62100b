// Sequences, new tokens and pages of a cache, as its kernels see them.  What lies in the arrays is cut off to what the tensors have room for.
#pragma once

#include "cache.h"

namespace ca {
namespace {

struct Sequence {
  int32_t first, count;   // rows of the packed tensors
  int32_t length, origin; // tokens, and those of the prompt
  int32_t base;           // tokens that are not new; below 0 where there are more new tokens than tokens
};

__device__ __forceinline__ Sequence sequence_at(const CacheArgs& a, int32_t s) {
  Sequence q;
  const int32_t to = a.starts[s + 1], from = a.starts[s], length = a.lengths[s], origin = a.origins ? a.origins[s] : 0;
  q.first = max(0, min(from, a.tokens));
  q.count = max(0, min(to, a.tokens) - q.first);
  q.length = max(0, min(length, a.table_width * a.page_tokens));
  q.origin = max(0, min(origin, q.length));
  q.base = q.length - q.count;
  return q;
}

// x / by, in 32 bits; plain tokens and ungrouped heads divide by one.
__device__ __forceinline__ int32_t divided(int32_t x, int32_t by) { return by == 1 ? x : (int32_t)((uint32_t)x / (uint32_t)by); }

// The same in 64 bits, of which most calls need 32.
__device__ __forceinline__ int64_t divided64(int64_t x, int64_t by) { return (uint64_t)(x | by) >> 32 ? x / by : (int64_t)((uint32_t)x / (uint32_t)by); }

// Page of a token that the table has an entry for, -1 where it is not there.
__device__ __forceinline__ int32_t page_at(const CacheArgs& a, int32_t s, int32_t token) {
  const int32_t page = a.table[(int64_t)s * a.table_width + divided(token, a.page_tokens)];
  return page >= 0 && page < a.num_pages ? page : -1;
}

// Row of a page's slot in [page][head][slot].
__device__ __forceinline__ int64_t cache_row(const CacheArgs& a, int32_t page, int32_t head, int32_t slot) {
  return ((int64_t)page * a.kv_heads + head) * a.page_tokens + slot;
}

}  // namespace
}  // namespace ca
