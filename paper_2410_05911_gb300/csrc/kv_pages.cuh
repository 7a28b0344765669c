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

// The row of head 0 that holds row r of a call's tokens (those of further heads follow page_size rows apart), -1 for a row of no sequence and a
// token without a page.  rows: s.rows, or a copy.  The rows of a sequence are its last tokens.
__device__ __forceinline__ int64_t token_row(const KvPages &c, const KvSequences &s, const int32_t *rows, int r) {
  int b = r;
  int64_t after = 1;  // rows of the sequence from r on
  if (rows) {
    int lo = 0, hi = s.batch;  // the last b with rows[b] <= r
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (rows[mid + 1] <= r) lo = mid + 1;
      else hi = mid;
    }
    b = lo;
    if (b >= s.batch || rows[b] > r) return -1;
    after = static_cast<int64_t>(rows[b + 1]) - r;
  }
  const int64_t p = s.lengths[b] - after;
  if (p < 0 || p >= static_cast<int64_t>(s.columns) * c.page_size) return -1;
  const int position = static_cast<int>(p), column = position / c.page_size, page = s.table[static_cast<int64_t>(b) * s.ldt + column];
  if (page < 0 || page >= c.pages) return -1;
  return static_cast<int64_t>(page) * c.heads * c.page_size + (position - column * c.page_size);
}

}  // namespace aecct
