// paged.h -- addressing of the paged 4-bit cache in device code: which sequence
// a row belongs to, and where a token lies.  Whatever the device arrays of a
// batch hold, no place that these functions return lies outside the cache.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "serving.h"

namespace comet {

// The page of token `pos` of sequence b, or -1 for a hole.
__device__ inline int token_page(const PagedBatch& b, int seq, long long pos, int page_shift,
                                 int num_pages) {
  const long long i = pos >> page_shift;
  if (pos < 0 || i >= b.max_pages) return -1;
  const int page = b.block_table[(long long)seq * b.max_pages + i];
  return (unsigned)page < (unsigned)num_pages ? page : -1;
}

// A slab is the part of a page that one head has: page * kv_heads + head, below
// 2^31 (the interface refuses larger caches).  -1 for a page outside the cache.
__device__ inline int slab_of(const PagedCache& c, int head, int page) {
  return (unsigned)page < (unsigned)c.num_pages ? page * c.kv_heads + head : -1;
}

// Row of token `pos` in its slab among all rows of the cache; a hole reads the
// first slab.
__device__ inline long long slab_row(const PagedCache& c, int slab, int pos) {
  return ((long long)max(slab, 0) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
}

// Row of (page, head, slot) among all rows of the cache; pages of a long cache
// pass 32 bits.
__device__ inline long long cache_row(const PagedCache& c, int page, int head, long long pos) {
  const int slot = (int)(pos & ((1 << c.page_shift) - 1));
  return (((long long)page * c.kv_heads + head) << c.page_shift) + slot;
}

// Sequence and position of row m: the sequence is the number of ends
// row_start[1 ..] that are <= m, found by halving.  False for a row in no
// sequence.
__device__ inline bool find_row(const PagedBatch& b, int m, int* seq, long long* pos) {
  int lo = 0, hi = b.B;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (b.row_start[mid + 1] <= m)
      lo = mid + 1;
    else
      hi = mid;
  }
  if (lo >= b.B || b.row_start[lo] > m) return false;
  *seq = lo;
  *pos = (long long)b.seq_lens[lo] - b.row_start[lo + 1] + m;
  return true;
}

}  // namespace comet
