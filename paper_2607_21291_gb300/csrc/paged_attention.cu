// Attention of new tokens over a paged cache: which kernel runs.
#include "internal.h"

#include <algorithm>

namespace adadsf {

// Packed rows (tokens x query heads of a group) of a sequence up to which paged_rows.cu runs: it reads the cache
// once per 16 of them. us at 8 sequences of 4096 cached keys, 28 query heads on 4, that kernel and the one
// on tcgen05: 28 rows (4 tokens) 31 and 45, 63 rows (9 tokens) 47 and 46.
constexpr int kFewRows = 64;

size_t paged_attention_scratch(int dtype, const Paged& p) {
  return dtype == kBF16 ? std::max(paged_rows_scratch(p), paged_tc_scratch(p)) : paged_f32_scratch(p);
}

cudaError_t paged_attention(int dtype, const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch,
                            const Dev& dev) {
  if (dtype == kF32) return paged_f32(p, q, ld_q, out, sync, scratch, dev);
  // a group of more heads than a row tile of tcgen05 has lanes stays with the rows
  if ((int64_t)p.max_new * (p.Hq / p.Hkv) <= kFewRows || !paged_tc_takes(p)) return paged_rows(p, q, ld_q, out, sync, scratch, dev);
  return paged_tc(p, q, ld_q, out, sync, scratch, dev);
}

}  // namespace adadsf
