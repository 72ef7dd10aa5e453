// Attention of new tokens over a paged cache: which kernel runs.
#include "internal.h"

#include <algorithm>

namespace adadsf {

// Which bf16 calls paged_rows.cu takes, by packed rows of a sequence (tokens x query heads of a group), items (16 rows of
// a key/value head) and steps (an item's tiles of 64 keys), as the host can bound them: by the table's width, not by the
// lengths. It reads the cache once per 16 rows: up to 16 always, from an 8-bit cache up to 32, of which the other kernel
// converts blocks for 256 rows that are mostly empty. Beyond, while its steps take less than what paged_tc.cu
// needs besides its products (joining, and blocks of 128 rows that are not full), that is up to kFewSteps steps times features,
// for up to kFewRows rows, or for few items, which the other kernel would cut in many pieces.
// us, this kernel and that one, tables as wide as the sequences are long:
//   28 heads of 128 on 4    8 sequences of 4096, 4 tokens 26 and 36, 6 tokens 33 and 36, 9 tokens 43 and 40; 64 of 300, 9
//                           tokens 36 and 25; 16 of 16000, 4 tokens 160 and 114; 64 of 4096, 4 tokens 167 and 120
//     in 8 bits             4 tokens: 8 of 4096 34 and 45, 64 of 4096 181 and 203, 32 of 16000 330 and 361, 16 of 32000 327 and 360;
//                           6 tokens: 8 of 4096 44 and 45, 16 of 4096 76 and 64
//     one sequence          32 tokens on 300 13 and 16, on 4096 26 and 39; 64 on none 14 and 13; 128 on 300 26 and 20
//   12 heads of 64          32 sequences of 700, 32 tokens 39 and 53, 64 tokens 68 and 56; one of 500, 100 tokens 13 and 18
//     in 8 bits             32 of 700, 32 tokens 40 and 74; 32 of 4096, 20 tokens 161 and 231
// Under a table of 131072 tokens, one sequence's 12 tokens of 28 heads go to that kernel: on 300 12.3 where the cut table's 9.9, on
// 4096 31 where 19.
constexpr int kAnyRows = 16, kAnyRowsI8 = 32, kFewRows = 48;
constexpr int64_t kFewItems = 128, kFewSteps = 1 << 20;

size_t paged_attention_scratch(int dtype, const Paged& p) {
  return dtype == kBF16 ? std::max(paged_rows_scratch(p), paged_tc_scratch(p)) : paged_f32_scratch(p);
}

cudaError_t paged_attention(int dtype, const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch,
                            const Dev& dev) {
  if (dtype == kF32) return paged_f32(p, q, ld_q, out, sync, scratch, dev);
  const int64_t G = p.Hq / p.Hkv, rows = p.max_new * G;
  const int64_t items = std::min<int64_t>(p.Hkv * std::min(p.B * ((rows + 15) / 16), p.n_rows * G / 16 + p.B), 1 << 24);
  const int64_t steps = items * ((((int64_t)p.max_pages << p.page_log2) + 63) / 64);
  // a group of more heads than a row tile of tcgen05 has lanes stays with the rows
  if (rows <= (p.i8 ? kAnyRowsI8 : kAnyRows) || (steps * p.hd <= kFewSteps && (rows <= kFewRows || items <= kFewItems)) || !paged_tc_takes(p))
    return paged_rows(p, q, ld_q, out, sync, scratch, dev);
  return paged_tc(p, q, ld_q, out, sync, scratch, dev);
}

}  // namespace adadsf
