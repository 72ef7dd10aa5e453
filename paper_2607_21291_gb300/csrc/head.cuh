// Shared pieces of the losses at the LM head (head.cu, head_tc.cu).
//
// A row's targets are k classes with weights p, classes ascending (distillation) or one class
// of weight 1 (cross entropy). With z = l / T, l = h W^T, q = softmax(z) over all classes:
//   lse = log sum e^z,  loss = T^2 (sum p log p - sum p z_c + lse),  G = g T (q - p)
// and dH = G W, dW = G^T H. Rows without a target are taken out first: the others are packed
// into a buffer (count of them on the device), and everything below runs on packed rows.
#pragma once

#include <limits.h>

#include "common.cuh"
#include "internal.h"

namespace adadsf {

constexpr int kHeadChunk = 8, kHeadChunkF32 = 4;   // blocks of 64 k of a logit that share an accumulator, in every kernel (see head_tc.cu)
constexpr int kHeadZeroPad = 64;   // rows past the last packed one, up to a multiple of this, are zero in the packed copy

// fp32 numbers as sums of three bf16 numbers, their leading 8 bits, the next 8 and the last: the next part of a (low
// half) and b (high half), which keep what it leaves. Exact; an infinity becomes NaN.
__device__ __forceinline__ uint32_t next_parts(float& a, float& b) {
  const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
  a -= __uint_as_float(ua & 0xffff0000u);
  b -= __uint_as_float(ub & 0xffff0000u);
  return __byte_perm(ua, ub, 0x7632);
}

// Parts of the two operands of each product of an fp32 product's parts.
constexpr int kHeadTerms = 6;
__device__ __forceinline__ int head_part_a(int term) { return (0x001102 >> (4 * term)) & 3; }   // 2 0 1 1 0 0
__device__ __forceinline__ int head_part_b(int term) { return (0x010120 >> (4 * term)) & 3; }   // 0 2 1 0 1 0

// First of a row's k ascending classes that is not below c0.
__device__ __forceinline__ int first_class(const int32_t* cls, int k, int c0) {
  int lo = 0, hi = k;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (cls[mid] < c0) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// The i-th of 32 registers (31 selects; indexing would move all of them to memory).
__device__ __forceinline__ float pick32(const uint32_t (&r)[32], int i) {
  uint32_t a[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) a[j] = (i & 16) ? r[j + 16] : r[j];
#pragma unroll
  for (int j = 0; j < 8; ++j) a[j] = (i & 8) ? a[j + 8] : a[j];
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = (i & 4) ? a[j + 4] : a[j];
#pragma unroll
  for (int j = 0; j < 2; ++j) a[j] = (i & 2) ? a[j + 2] : a[j];
  return __uint_as_float((i & 1) ? a[1] : a[0]);
}

}  // namespace adadsf
