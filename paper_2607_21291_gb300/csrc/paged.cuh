// Device side of a paged cache (adadsf_paged_cache, adadsf_paged_batch): where a
// sequence's tokens lie, with every count clamped into range and reported.
#pragma once

#include "common.cuh"
#include "internal.h"

namespace adadsf {

// The rows and cached tokens of one sequence.
struct PagedSeq {
  int64_t row0;   // first packed row
  int n, len;     // rows, cached tokens
};
__device__ __forceinline__ PagedSeq paged_seq(const Paged& p, int b, int* err) {
  const int s0 = p.starts[b], s1 = p.starts[b + 1], l = p.lens[b];
  const int rows = (int)p.n_rows, room = p.max_pages << p.page_log2;
  PagedSeq q;
  const int a = min(max(s0, 0), rows), e = min(max(s1, a), rows);
  q.row0 = a;
  q.n = min(e - a, p.max_new);
  q.len = min(max(l, 0), room);
  if (a != s0 || a + q.n != s1 || q.len != l) set_device_error(err, DEVERR_INDEX);
  return q;
}
// Number of starts[1 .. B] at or below `row`: the sequence a packed row belongs to
// (B: none). Whole warp; 32 boundaries of every level are read at once.
__device__ __forceinline__ int paged_find(const Paged& p, int64_t row, int lane) {
  int lo = 0, n = p.B;   // the answer is in [lo, lo + n]
  while (n > 0) {
    const int step = (n + 31) / 32;
    const int i = lo + (lane + 1) * step;   // boundary after (lane + 1) steps
    const bool below = (lane + 1) * step <= n && p.starts[i] <= row;
    const int c = __popc(__ballot_sync(0xffffffffu, below));
    lo += c * step;
    n = min(step - 1, n - c * step);
  }
  return lo;
}
// Page of the token at `place` (in [0, len)) of sequence b, or -1 if its number is
// out of range (reported).
__device__ __forceinline__ int paged_page(const Paged& p, int b, int place, int* err) {
  const int page = p.table[(int64_t)b * p.max_pages + (place >> p.page_log2)];
  if ((unsigned)page < (unsigned)p.n_pages) return page;
  set_device_error(err, DEVERR_INDEX);
  return -1;
}
// Index of a token's vector of head h: times hd its first feature, itself its scale.
__device__ __forceinline__ int64_t paged_vec(const Paged& p, int page, int place, int h) {
  return (((int64_t)page * p.Hkv + h) << p.page_log2) + (place & ((1 << p.page_log2) - 1));
}

}  // namespace adadsf
