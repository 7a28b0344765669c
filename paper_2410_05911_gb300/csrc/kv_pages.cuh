// kv_pages.cuh -- where a paged cache holds a token: shared by the kernels that write, read and attend to it.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "aecct_internal.h"

namespace aecct {

// the tokens of sequence b that its pages can hold
__device__ __forceinline__ int sequence_length(const KvSequences &s, int b, int page_size) {
  const int n = s.lengths[b], most = s.columns * page_size;
  return n < 0 ? 0 : n < most ? n : most;
}

// place of position p (0 <= p < sequence_length) of sequence b, counted over the pages' tokens of one head: page * page_size +
// offset; -1 where there is no such page
__device__ __forceinline__ int64_t token_place(const KvPages &c, const KvSequences &s, int b, int p) {
  const int column = p / c.page_size;
  const int page = s.table[static_cast<int64_t>(b) * s.ldt + column];
  if (page < 0 || page >= c.pages) return -1;
  return static_cast<int64_t>(page) * c.page_size + (p - column * c.page_size);
}

// the row (of all heads' rows) of a place and a head: [pages][heads][page_size]
__device__ __forceinline__ int64_t cache_row(const KvPages &c, int64_t place, int head) {
  const int64_t page = place / c.page_size;
  return (page * c.heads + head) * c.page_size + (place - page * c.page_size);
}

// The page and place in it of row r of a call's tokens, -1 for a row of no sequence and a token without a page.  The rows of a
// sequence are its last tokens.
__device__ __forceinline__ int64_t row_place(const KvPages &c, const KvSequences &s, int r) {
  int b = r;
  int64_t after = 1;  // rows of the sequence from r on
  if (s.rows) {
    int lo = 0, hi = s.batch;  // the last b with rows[b] <= r
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s.rows[mid + 1] <= r) lo = mid + 1;
      else hi = mid;
    }
    b = lo;
    if (b >= s.batch || s.rows[b] > r) return -1;
    after = static_cast<int64_t>(s.rows[b + 1]) - r;
  }
  const int64_t p = s.lengths[b] - after;
  if (p < 0 || p >= static_cast<int64_t>(s.columns) * c.page_size) return -1;
  return token_place(c, s, b, static_cast<int>(p));
}

}  // namespace aecct
