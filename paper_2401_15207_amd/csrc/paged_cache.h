// A paged cache as the kernels see it: where a sequence's new rows are and which page holds a token.  Everything that comes from device memory
// is brought into range here, so that no content of those arrays leads past a buffer.
#pragma once
#include "common.h"
#include "kernels.h"

namespace hift {

struct CacheSeq {
  int64_t row0;  // first of its new rows
  int fresh;     // new rows, at most max_new
  int cached;    // tokens before them
  int total;     // tokens that there are with them, as far as pages reach
};

__device__ __forceinline__ int cache_capacity(const CacheView& c) { return c.max_pages << c.page_shift; }

__device__ __forceinline__ CacheSeq cache_seq(const CacheView& c, int s, int64_t rows, int max_new) {
  const int a = min(max(c.starts[s], 0), (int)rows), b = min(max(c.starts[s + 1], a), (int)rows);
  const int cap = cache_capacity(c);
  CacheSeq of;
  of.row0 = a;
  of.fresh = min(b - a, max_new);
  of.cached = min(max(c.lengths[s], 0), cap);
  of.total = min(of.cached + of.fresh, cap);
  return of;
}

// The page of sequence s that holds token `pos` (>= 0), or -1.
__device__ __forceinline__ int cache_page(const CacheView& c, int s, int pos) {
  const int i = pos >> c.page_shift;
  if (i >= c.max_pages) return -1;
  // no kernel writes page numbers: with a uniform index a scalar load, which loads in flight to LDS do not wait for
  typedef const __attribute__((address_space(4))) int32_t* Constant;
  const int page = reinterpret_cast<Constant>(reinterpret_cast<uintptr_t>(c.pages))[(int64_t)s * c.pages_ld + i];
  return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}
// The same for a token of the lane's own.
__device__ __forceinline__ int cache_page_any(const CacheView& c, int s, int pos) {
  const int i = pos >> c.page_shift;
  if (i >= c.max_pages) return -1;
  const int page = c.pages[(int64_t)s * c.pages_ld + i];
  return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}

}  // namespace hift
