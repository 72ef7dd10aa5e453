// Attention of new tokens over a paged cache: which kernel runs.
#include "internal.h"

#include <algorithm>

namespace adadsf {

// Packed rows (tokens x query heads of a group) of a sequence up to which paged_rows.cu runs: it reads the cache
// once per 16 of them. us at 8 sequences of 4096 cached keys, 28 query heads on 4, that kernel and the one
// on tcgen05: 28 rows (4 tokens) 31 and 45, 63 rows (9 tokens) 47 and 46.
constexpr int kFewRows = 64;
// Beyond them it runs while 16 rows of a key/value head make no more items than these, and these and their tiles of 64
// keys no more steps: few items in many pieces cost the other kernel their joining. us, that kernel and the one
// on tcgen05, 28 heads on 4: 32 tokens on 300 13 and 16, on 4096 26 and 39; 64 on 0 14 and 13; 128 on 300 (224 items) 26
// and 20; 20 on 20000 (11268 steps) 51 and 54; 12 heads of 64: 100 on 500 13 and 18, in 8 bits 13 and 23.
constexpr int64_t kFewItems = 128, kFewSteps = 8192;

size_t paged_attention_scratch(int dtype, const Paged& p) {
  return dtype == kBF16 ? std::max(paged_rows_scratch(p), paged_tc_scratch(p)) : paged_f32_scratch(p);
}

cudaError_t paged_attention(int dtype, const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch,
                            const Dev& dev) {
  if (dtype == kF32) return paged_f32(p, q, ld_q, out, sync, scratch, dev);
  const int64_t G = p.Hq / p.Hkv;
  const int64_t items = p.Hkv * std::min(p.B * ((p.max_new * G + 15) / 16), p.n_rows * G / 16 + p.B);   // at most
  const int64_t steps = items * ((((int64_t)p.max_pages << p.page_log2) + 63) / 64);
  // a group of more heads than a row tile of tcgen05 has lanes stays with the rows
  if (p.max_new * G <= kFewRows || (items <= kFewItems && steps <= kFewSteps) || !paged_tc_takes(p))
    return paged_rows(p, q, ld_q, out, sync, scratch, dev);
  return paged_tc(p, q, ld_q, out, sync, scratch, dev);
}

}  // namespace adadsf
