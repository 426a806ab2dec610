// Where tokens of a sequence are: device code of the kernels that use the paged
// cache.  Lengths, starts and pages come from device memory, so nothing about
// them is taken for granted: what lies outside the tensors is never touched.
#pragma once

#include "cache.h"

namespace syncgb {
namespace paged {

// The sequence that has `row`: the last s with starts[s] <= row, if row <
// starts[s + 1] too; -1: none.
__device__ __forceinline__ int sequence_of(const CacheArgs& a, int row) {
  if (!a.starts) return row < a.n_seqs ? row : -1;
  int lo = 0, hi = a.n_seqs;                                // starts[lo] <= row < starts[hi], as far as they rise
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (mid < a.n_seqs && __ldg(a.starts + mid) <= row) lo = mid;
    else hi = mid - 1;
  }
  return a.n_seqs > 0 && __ldg(a.starts + lo) <= row && row < __ldg(a.starts + lo + 1) ? lo : -1;
}

// The place of a token in the cache, counted in tokens of one head: page number
// times page size plus the offset; -1 where the table has no such page.
__device__ __forceinline__ int64_t place_of(const CacheArgs& a, int s, int64_t pos) {
  if (pos < 0 || pos >> a.page_shift >= a.max_pages) return -1;
  const int page = __ldg(a.table + s * a.table_stride + (pos >> a.page_shift));
  if ((unsigned)page >= (unsigned)a.n_pages) return -1;
  return ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
}
// The row of a head of that token, counted in rows of the cache.
__device__ __forceinline__ int64_t row_of(const CacheArgs& a, int64_t place, int head) {
  const int64_t page = place >> a.page_shift;
  return ((page * a.kv_heads + head) << a.page_shift) + (place & ((1 << a.page_shift) - 1));
}

// Word of a row of 4-bit codes that has entries 8 i .. 8 i + 7, in a row of g
// groups: word g c + w has entries 32 w + 8 c on, so that a quarter of a row has
// a quarter of every group (what a thread of the attention kernel takes).
__device__ __forceinline__ int word_of(int i, int g) { return g * (i % 4) + i / 4; }

}  // namespace paged
}  // namespace syncgb
