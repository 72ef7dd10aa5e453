// The next token of a row of logits by temperature, top-k, top-p, min-p and a given
// random number (adadsf_sample).
//
// A cluster of CTAs holds one row in shared memory as ordered 32-bit keys (larger
// key = larger logit), each CTA a contiguous slice, each thread a contiguous chunk of
// it (an odd number of words, so that a warp's chunks spread over the banks), so logits
// are read from memory once. Kept tokens are a prefix of the descending order, so a
// cut (key, number of equal ones kept) describes them. A cut is found by histograms of counts
// (top-k) or of weights (top-p): every CTA makes its own, then adds up all of them through distributed
// shared memory and finds the same bin. The first histogram's bins are even in the logits'
// distance from the largest (bins of the keys' leading bits, four to an octave, put the bulk of a row
// into a few of them, and its atomics into one queue), the next ones' even in the keys of the bin
// found, down to one key. Weights are whole multiples of 2^-40 of the largest, so
// their sums do not depend on order, and neither does the token.
// For top-k up to the number of warps, keys below the smallest of the warps' largest ones are out at once. When
// few keys are left (kSmList), they move to one CTA, whose rounds take a third of the time of the cluster's.
// Few rows are bound by the latency of those rounds (two to eight, 2 us each over the cluster), many
// rows by the instructions of the passes over the keys, half of them comparisons and logic on a pipe of half
// rate. Measured: one row of 50304 bf16 5 us greedy, 11 with top-k 50, 15 with top-p 0.9; 16 rows of 152064 fp32 of
// mixed settings 31 us; 256 of 151936 bf16 173 us (54 greedy, 83 with top-k 50, 277 with top-p 0.9).
#include <math.h>

#include <type_traits>

#include "common.cuh"

namespace adadsf {
namespace {

typedef unsigned long long u64;

constexpr int kSmThreads = 512;
constexpr int kSmWarps = kSmThreads / 32;
constexpr int kSmBinsLog2 = 9, kSmBins = 1 << kSmBinsLog2;
static_assert(kSmBins == kSmThreads, "a thread a bin");
constexpr int kSmMostChunk = 97;          // words of a thread: 8 x 512 x 97 tokens
constexpr int kSmMostCluster = 8;
constexpr int kSmSmem = kSmThreads * kSmMostChunk * 4 + 16;
static_assert((uint64_t)kSmThreads * kSmMostChunk << 14 < 1ull << 31, "14 bits of every key of a CTA, and top-k's equals' upper ones");
static_assert(kSmMostCluster * kSmThreads * kSmMostChunk == kSampleMaxV, "the limit that the header states");
// Keys that a search leaves are gathered in one CTA where they are this few.
constexpr int kSmList = 3 * kSmThreads;
constexpr uint32_t kSmNone = 0x007fffffu; // key of -infinity, of NaN and of padding
// First bins: even in the distance from the largest logit (or from z = 0) to this, the last one takes the
// rest (weights end at 28).
constexpr float kSmEnd = 32.f, kSmBinsPer = (kSmBins - 1) / kSmEnd;
constexpr float kSmUnit = 1099511627776.f;   // 2^40

__device__ __forceinline__ uint32_t key_of(float x) {
  // -0 equals 0; a NaN is never drawn, as -infinity is not
  const uint32_t u = __float_as_uint(fmaxf(__fadd_rn(x, 0.f), -INFINITY));
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float((~(uint32_t)((int32_t)key >> 31) | 0x80000000u) ^ key);
}
// A weight w in [0, 1] as whole multiples of 2^-40, to the nearest one, ties to even: hi 2^20 + lo, hi and lo up to 2^20. Sums
// with 2^3 and 2^-17 round to multiples of 2^-20 and 2^-40 and leave them in their low bits: no conversions,
// which go through a unit a sixteenth as wide, nor 64-bit shifts.
struct SmWeight {
  uint32_t a, b;   // bits of the two sums
  __device__ __forceinline__ uint32_t hi() const { return a - 0x41000000u; }
  __device__ __forceinline__ uint32_t lo() const { return b - 0x37000000u; }
  __device__ __forceinline__ u64 whole() const { return ((u64)hi() << 20) + lo(); }
};
__device__ __forceinline__ SmWeight weight_of(float w) {
  const float a = __fadd_rz(w, 8.f), rest = __fsub_rn(w, __fsub_rn(a, 8.f));   // below 2^-20, exact
  return SmWeight{__float_as_uint(a), __float_as_uint(__fadd_rn(rest, 7.62939453125e-06f))};
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ u64 ld_cluster_u64(uint32_t addr) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

struct SampleShared {
  // Histograms: counts in part 0, or weights in 14, 14 and the other bits: a CTA's keys do not fill a word with
  // 14 bits each, so that an addition needs no carry and nothing waits for it. Rounds over the cluster
  // take turns with two of everything that other CTAs read, so one barrier a round is enough.
  uint32_t part[2][3][kSmBins];        // or the gathered keys, as they come in
  u64 total[2];                        // this CTA's total
  u64 bins[2][kSmBins];                // sums over the cluster of this CTA's share of the bins, or the gathered keys' indices
  u64 warp[kSmWarps];                  // block scan
  u64 found_before, found_in, found_target;
  uint32_t found_bin;
  uint32_t most, least;                // this CTA's largest key, the smallest of its warps' largest ones; read by the cluster
  uint32_t index;                      // written by the CTA that finds it
};

// Sum of v over the block's threads before this one; *all: over all of them.
__device__ __forceinline__ u64 block_before(u64 v, SampleShared& s, u64* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 up = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += up;
  }
  __syncthreads();   // the last call's sums are read
  if (lane == 31) s.warp[warp] = inc;
  __syncthreads();
  u64 sums = lane < kSmWarps ? s.warp[lane] : 0;
#pragma unroll
  for (int o = 1; o < kSmWarps; o <<= 1) {
    const u64 up = __shfl_up_sync(0xffffffffu, sums, o);
    if (lane >= o) sums += up;
  }
  *all = __shfl_sync(0xffffffffu, sums, kSmWarps - 1);
  const u64 base = __shfl_sync(0xffffffffu, sums, warp ? warp - 1 : 0);
  return (warp ? base : 0) + inc - v;
}

// The CTAs that hold the row's keys: a cluster, or one.
__device__ __forceinline__ void row_sync(uint32_t n) {
  if (n > 1) cluster_sync();
  else __syncthreads();
}

// block_before over the threads of n CTAs in order of their slices. A round of the cluster.
__device__ __forceinline__ u64 row_before(u64 v, SampleShared& s, int& round, u64* all, uint32_t n, uint32_t rank) {
  u64 mine;
  u64 before = block_before(v, s, &mine);
  *all = mine;
  if (n == 1) return before;
  const int q = round++ & 1;
  if (threadIdx.x == 0) s.total[q] = mine;
  cluster_sync();
  const uint32_t lane = threadIdx.x & 31;
  const u64 t = lane < n ? ld_cluster_u64(map_to_cta(smem_u32(&s.total[q]), lane)) : 0;
  u64 lower = lane < rank ? t : 0, sum = t;
#pragma unroll
  for (int o = 1; o < kSmMostCluster; o <<= 1) {   // the first lanes, a CTA each
    lower += __shfl_xor_sync(0xffffffffu, lower, o);
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
  }
  *all = __shfl_sync(0xffffffffu, sum, 0);
  return before + __shfl_sync(0xffffffffu, lower, 0);
}

// The smallest whole number whose double is `target` or more: compared with it, whole sums need no doubles.
__device__ __forceinline__ u64 whole_target(double target) {
  u64 v = (u64)ceil(target);
  while (v > 0 && (double)(v - 1) >= target) --v;
  return v;
}

// Adds up the cluster's histograms number `q`, whose bins run from the largest keys down, and finds the
// first bin that takes the running sum, from `base` on, to `target` or more. frac < 1: the
// target is frac times the sum of all bins (at least 1), left in s.found_target. Results in s.found_*.
// Where no bin does, it is the last one, which leaves everything in.
// Each CTA adds up a share of the bins and all read the sums (every CTA reading every histogram took 8 us
// a round, 11-bit ones 25: 16 words a thread cross the cluster's network slowly).
template <bool WEIGHTS>
__device__ __forceinline__ void find_bin(SampleShared& s, int q, u64 base, u64 target, double frac, uint32_t n, uint32_t rank) {
  const uint32_t share = kSmBins / n;
  const int tid = threadIdx.x;
  row_sync(n);   // every CTA's histogram is complete
  u64 v;
  if (n > 1) {
    const uint32_t c = tid & (n - 1), bin = rank * share + tid / n;
    v = ld_cluster_u32(map_to_cta(smem_u32(&s.part[q][0][bin]), c));
    if (WEIGHTS) {
      v += (u64)ld_cluster_u32(map_to_cta(smem_u32(&s.part[q][1][bin]), c)) << 14;
      v += (u64)ld_cluster_u32(map_to_cta(smem_u32(&s.part[q][2][bin]), c)) << 28;
    }
    for (uint32_t o = 1; o < n; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (c == 0) s.bins[q][tid / n] = v;
    cluster_sync();
    v = ld_cluster_u64(map_to_cta(smem_u32(&s.bins[q][tid & (share - 1)]), tid / share));
  } else {
    v = s.part[q][0][tid];
    if (WEIGHTS) v += ((u64)s.part[q][1][tid] << 14) + ((u64)s.part[q][2][tid] << 28);
  }
  u64 all;
  const u64 run = base + block_before(v, s, &all);
  if (frac < 1.0) {
    if (tid == 0) s.found_target = whole_target(fmax(frac * (double)all, 1.0));
    __syncthreads();
    target = s.found_target;
  }
  if (run < target && (run + v >= target || tid == kSmBins - 1)) {
    s.found_bin = tid;
    s.found_before = run;
    s.found_in = v;
  }
  __syncthreads();
}

// Four consecutive elements, 16 or 8 aligned bytes.
__device__ __forceinline__ uint4 keys_of4(const float* p) {
  const float4 v = __ldg(reinterpret_cast<const float4*>(p));
  return make_uint4(key_of(v.x), key_of(v.y), key_of(v.z), key_of(v.w));
}
__device__ __forceinline__ uint4 keys_of4(const bf16* p) {
  const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
  return make_uint4(key_of(__uint_as_float(v.x << 16)), key_of(__uint_as_float(v.x & 0xffff0000u)),
                    key_of(__uint_as_float(v.y << 16)), key_of(__uint_as_float(v.y & 0xffff0000u)));
}

template <typename T>
__global__ void __launch_bounds__(kSmThreads, 2) sample_kernel(const Sample a, int chunk) {
  constexpr int KS = sizeof(T) == 2 ? 16 : 0;        // bits of a key that its type leaves alone
  extern __shared__ __align__(16) uint32_t raw[];    // [kSmThreads][chunk], shifted by up to three words
  __shared__ __align__(16) SampleShared s;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31;
  uint32_t n_cta = cluster_nctarank(), rank = cluster_ctarank();   // 1 or 8; once the row's keys are gathered, 1 and 0
  const int row = blockIdx.x / n_cta;
  const int slice = kSmThreads * chunk, i0 = (int)rank * slice;
  const T* x = static_cast<const T*>(a.logits) + (int64_t)row * a.ld + i0;
  // groups of four elements that are aligned in memory, aligned in shared memory too
  const int shift = (int)((reinterpret_cast<uintptr_t>(x) / sizeof(T)) & 3);
  uint32_t* keys = raw + shift;
  const uint32_t* index = nullptr;     // of gathered keys
  const int there = min(max(a.V - i0, 0), slice);
  uint32_t most = 0;
  const int g0 = shift ? 1 : 0, g1 = (there + shift) / 4;   // whole groups
#pragma unroll 8
  for (int g = g0 + tid; g < g1; g += kSmThreads) {
    const uint4 k = keys_of4(x + 4 * g - shift);
    *reinterpret_cast<uint4*>(raw + 4 * g) = k;
    most = max(max(most, max(k.x, k.y)), max(k.z, k.w));
  }
  if (tid < 8) {   // up to three elements on either side
    const int i = tid < 4 ? tid : max(4 * g1 - shift, 4 * g0 - shift) + tid - 4;
    if (tid < 4 ? i < 4 * g0 - shift && i < there : i < there) {
      keys[i] = key_of(Elem<T>::to_f(x[i]));
      most = max(most, keys[i]);
    }
  }
  for (int i = there + tid; i < slice; i += kSmThreads) keys[i] = kSmNone;
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 0) s.warp[tid >> 5] = most;
  __syncthreads();
  if (tid == 0) {
    uint32_t least = most;
    for (int w = 1; w < kSmWarps; ++w) {
      most = max(most, (uint32_t)s.warp[w]);
      least = min(least, (uint32_t)s.warp[w]);
    }
    s.most = most;
    s.least = least;
    s.index = 0xffffffffu;
  }
  cluster_sync();
  // a lane a CTA: loads from other CTAs one behind the other take a third of a microsecond each
  most = __reduce_max_sync(0xffffffffu, lane < (int)n_cta ? ld_cluster_u32(map_to_cta(smem_u32(&s.most), lane)) : 0u);
  const uint32_t least = __reduce_min_sync(0xffffffffu, lane < (int)n_cta ? ld_cluster_u32(map_to_cta(smem_u32(&s.least), lane)) : ~0u);

  const uint32_t* own = keys + tid * chunk;
  const float t = a.temperature ? a.temperature[row] : 1.f;
  const float inv = 1.f / t, top = value_of(most);
  auto logit_of = [&](uint32_t k) { return k == most ? 0.f : __fmul_rn(__fsub_rn(value_of(k), top), inv); };
  // exp(z): 0 of kSmNone, whose z is -infinity or NaN, as it is of an infinite logit under an infinite temperature
  auto chance = [&](uint32_t k) -> float { return fmaxf(expf(logit_of(k)), 0.f); };
  // f(i, keys i to i + 3) over the thread's keys, behind the last one kSmNone, where one is `low` or above: four chains
  // of arithmetic side by side
  auto by_four = [&](uint32_t low, auto f) {
#pragma unroll 1
    for (int i = 0; i < chunk; i += 4) {
      uint32_t k4[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) k4[j] = i + j < chunk ? own[i + j] : kSmNone;
      if (max(max(k4[0], k4[1]), max(k4[2], k4[3])) >= low) f(i, k4);
    }
  };
  auto weight = [&](float w) -> u64 { return weight_of(w).whole(); };
  int round = 0;
  const int k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.f;
  const float floor_p = a.min_p ? a.min_p[row] : 0.f;
  const bool by_k = k > 0 && k < a.V, by_p = top_p < 1.f;
  // The first round of a search leaves the keys that can be kept, from low_key on, and among them the ones of
  // the bin that it found (keys from low to high): a bit for each of the thread's. Only those are looked at again.
  uint32_t low_key = 0, can[4] = {0, 0, 0, 0}, in_bin[4] = {0, 0, 0, 0};
  auto mark_from = [&](uint32_t low) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t above = 0;
      const int n = min(32, chunk - 32 * w);
#pragma unroll 4
      for (int i = 0; i < n; ++i) above |= (uint32_t)(own[32 * w + i] >= low) << i;
      can[w] = above;
    }
    low_key = low;
  };
  auto mark_keys = [&](uint32_t low, uint32_t high) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t above = 0, in = 0;
      const int n = min(32, chunk - 32 * w);
#pragma unroll 4
      for (int i = 0; i < n; ++i) {
        const uint32_t k = own[32 * w + i];
        above |= (uint32_t)(k >= low) << i;
        in |= (uint32_t)(k >= low && k <= high) << i;
      }
      can[w] = above;
      in_bin[w] = in;
    }
    low_key = low;
  };
  // f(g(i, own[i])) for the marked keys one by one
  auto each_of = [&](const uint32_t (&marks)[4], auto g, auto f) {
#pragma unroll 1
    for (int w = 0; w < 4; ++w)
      for (uint32_t m = w == 0 ? marks[0] : w == 1 ? marks[1] : w == 2 ? marks[2] : marks[3]; m; m &= m - 1)
        f(g(32 * w + __ffs(m) - 1, own[32 * w + __ffs(m) - 1]));
  };
  auto few = [&]() {   // whether the warp's keys that can be kept are few
    return low_key && !__any_sync(0xffffffffu, 3 * (__popc(can[0]) + __popc(can[1]) + __popc(can[2]) + __popc(can[3])) > chunk);
  };
  // Where, in the slice, a running sum passes `mark`, if that is in this warp's part: `before` and `sum` are
  // each thread's, value(i) the summands. The warp takes the thread's chunk 32 at a time. -1: elsewhere.
  auto walk = [&](u64 before, u64 sum, u64 mark, auto value) -> int {
    const unsigned has = __ballot_sync(0xffffffffu, before <= mark && mark < before + sum);
    if (!has) return -1;
    const int from = __ffs(has) - 1;
    u64 run = __shfl_sync(0xffffffffu, before, from);
    const int first = ((tid & ~31) + from) * chunk;
    for (int i = 0;; i += 32) {
      u64 inc = i + lane < chunk ? value(first + i + lane) : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      const unsigned past = __ballot_sync(0xffffffffu, run + inc > mark);
      if (past) return first + i + __ffs(past) - 1;
      if (i + 32 >= chunk) return first + chunk - 1;   // not reached: the sums say that it is here
      run += __shfl_sync(0xffffffffu, inc, 31);
    }
  };
  auto index_of = [&](int i) -> uint32_t { return index ? index[i] : (uint32_t)(i0 + i); };   // of number i of the slice
  // Where the keys that can be kept are few, they move to the first CTA in the vocabulary's order, which goes on alone: its
  // rounds need no cluster and take a third of the time. false: the others, which are done. Marks are to be made again.
  auto gather = [&]() -> bool {
    if (n_cta == 1) return true;
    const int mine = __popc(can[0]) + __popc(can[1]) + __popc(can[2]) + __popc(can[3]);
    u64 all;
    uint32_t at = (uint32_t)row_before((u64)mine, s, round, &all, n_cta, rank);
    if (all > kSmList) return true;
    const uint32_t to_key = map_to_cta(smem_u32(&s.part[0][0][0]), 0), to_index = map_to_cta(smem_u32(&s.bins[0][0]), 0);
    each_of(can, [&](int i, uint32_t key) { return make_uint2(key, (uint32_t)(i0 + tid * chunk + i)); }, [&](const uint2& a) {
      st_cluster_u32(to_key + 4 * at, a.x);
      st_cluster_u32(to_index + 4 * at, a.y);
      ++at;
    });
    cluster_sync();
    if (rank != 0) return false;
    n_cta = 1;
    chunk = ((int)all + kSmThreads - 1) / kSmThreads | 1;
    keys = raw;
    for (int i = tid; i < kSmThreads * chunk; i += kSmThreads) keys[i] = i < (int)all ? (&s.part[0][0][0])[i] : kSmNone;
    own = keys + tid * chunk;
    index = reinterpret_cast<const uint32_t*>(&s.bins[0][0]);
    __syncthreads();
    return true;
  };
  // index of the n-th (from 1) key equal to k in the order of the vocabulary, in every CTA
  auto nth = [&](uint32_t k, u64 n) -> uint32_t {
    int c = 0;
    if (few()) {
      each_of(can, [&](int, uint32_t key) { return (int)(key == k); }, [&](int one) { c += one; });
    } else {
#pragma unroll 4
      for (int i = 0; i < chunk; ++i) c += own[i] == k;
    }
    u64 all;
    const u64 before = row_before((u64)c, s, round, &all, n_cta, rank);
    const int i = walk(before, (u64)c, n - 1, [&](int i) -> u64 { return keys[i] == k; });
    if (i >= 0 && lane < (int)n_cta) st_cluster_u32(map_to_cta(smem_u32(&s.index), lane), index_of(i));
    row_sync(n_cta);
    return s.index;
  };

  if (most <= kSmNone) {   // nothing to draw
    if (rank == 0 && tid == 0) {
      a.token[row] = -1;
      if (a.logprob) a.logprob[row] = -INFINITY;
    }
    cluster_sync();        // no CTA leaves while another reads its shared memory
    return;
  }
  if (!(t > 0.f)) {
    const uint32_t i = nth(most, 1);
    if (rank == 0 && tid == 0) {
      a.token[row] = (int32_t)i;
      if (a.logprob) a.logprob[row] = 0.f;
    }
    return;
  }

  // ---- the cut: keys above cut_key, and the first cut_ties of those equal to it
  uint32_t cut_key = 0;
  u64 cut_ties = ~0ull;       // ~0: all
  bool some_ties = false;     // fewer than there are
  bool gone = false;          // the keys went to another CTA
  // One search. key_in: whether a key takes part, none below least_in does; more: weight of `more_key` beside those (0: none); target: as
  // find_bin takes it. Out: the key, and in s.found_* the sums before and of it.
  // Weights of keys below tail_key go into the last bin together.
  auto search = [&](auto weights_c, auto key_in, uint32_t least_in, uint32_t more_key, u64 more, u64 target, double frac, uint32_t tail_key) -> uint32_t {
    constexpr bool W = decltype(weights_c)::value;
    const float from = fminf(top, 3.4e38f), per = kSmBinsPer;
    auto bin0 = [&](uint32_t k) -> int {   // falls with the key, slowly or not at all
      const float d = __fsub_rn(from, value_of(k)), e = W ? __fmul_rn(d, inv) : d;
      const float at = fminf(fmaxf(__fmul_rn(e, per), 0.f), (float)(kSmBins - 1));   // NaN (0 times infinity): 0
      return (int)(__float_as_uint(__fadd_rz(at, 8388608.f)) & 0x7fffffu);          // whole part, without a conversion
    };
    struct Put { int bin; SmWeight w; };   // bin < 0: takes no part
    auto put = [&](int q, const Put& a) {
      if (a.bin < 0) return;
      if (!W) {
        atomicAdd(&s.part[q][0][a.bin], 1u);
        return;
      }
      const uint32_t lo = a.w.lo(), hi = a.w.hi(), p0 = lo & 0x3fffu, p1 = (lo >> 14) + ((hi & 0xffu) << 6), p2 = hi >> 8;
      atomicAdd(&s.part[q][0][a.bin], p0);
      atomicAdd(&s.part[q][1][a.bin], p1);
      if (p2) atomicAdd(&s.part[q][2][a.bin], p2);
    };
    auto clear = [&]() -> int {   // the histogram of the next round
      const int q = round++ & 1;
#pragma unroll
      for (int i = 0; i < (W ? 3 : 1); ++i) s.part[q][i][tid] = 0;
      __syncthreads();
      return q;
    };
    auto put_whole = [&](int q, int bin, u64 w) {   // any weight
      if (bin < 0) return;
      atomicAdd(&s.part[q][0][bin], (uint32_t)w & 0x3fffu);
      atomicAdd(&s.part[q][1][bin], (uint32_t)(w >> 14) & 0x3fffu);
      atomicAdd(&s.part[q][2][bin], (uint32_t)(w >> 28));
    };
    int q = clear();
    uint32_t rest_hi = 0, rest_lo = 0;
    auto first = [&](uint32_t key, const SmWeight& w) {
      const bool in = key_in(key), tail = W && key < tail_key;
      if (W) {
        rest_hi += in && tail ? w.hi() : 0;
        rest_lo += in && tail ? w.lo() : 0;
      }
      if (in && !tail) put(q, Put{bin0(key), w});
    };
    auto worth = [&](uint32_t key) { return W ? weight_of(chance(key)) : SmWeight{0, 0}; };
    if (low_key) {
      each_of(can, [&](int, uint32_t key) { return key; }, [&](uint32_t key) { first(key, worth(key)); });
    } else {
      by_four(least_in, [&](int, const uint32_t (&k4)[4]) {
        SmWeight w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = worth(k4[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) first(k4[j], w[j]);
      });
    }
    if (W) {
      u64 rest = ((u64)rest_hi << 20) + rest_lo;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
      if (lane == 0) put_whole(q, kSmBins - 1, rest);
      if (more && rank == 0 && tid == 0) put_whole(q, bin0(more_key), more);
    }
    find_bin<W>(s, q, 0, target, frac, n_cta, rank);
    if (frac < 1.0) target = s.found_target;
    // keys that can lie in the bin, with room for roundings
    const int bin = (int)s.found_bin;
    const float unit = W ? t / per : 1.f / per;
    const float far = top - (float)(bin + 1) * unit, near = top - (float)bin * unit;
    const float room = 1e-5f * (fabsf(top) + fabsf(far) + (float)(bin + 2) * unit);
    uint32_t lo = far - room > -INFINITY && bin < kSmBins - 1 ? key_of(far - room) : 0u;
    uint32_t hi = near + room < INFINITY && bin > 0 ? min(key_of(near + room), most) : most;
    lo >>= KS;
    hi >>= KS;
    const uint32_t low = min(max(lo << KS, low_key), most), high = hi << KS | ((1u << KS) - 1);
    mark_keys(low, high);
    if (n_cta > 1 && (W || s.found_before + s.found_in <= kSmList)) {
      if (!gather()) {
        gone = true;
        return 0;
      }
      if (n_cta == 1) mark_keys(low, high);
    }
    while (lo < hi) {
      const int bits = max(0, 32 - __clz(hi - lo) - kSmBinsLog2);   // (hi - lo) >> bits is below kSmBins
      const u64 before = s.found_before;
      auto bin_of = [&](uint32_t k) -> int {
        return (k >> KS) >= lo && (k >> KS) <= hi && bin0(k) == bin ? (int)((hi - (k >> KS)) >> bits) : -1;
      };
      q = clear();
      each_of(in_bin, [&](int, uint32_t key) {
        const int at = key_in(key) ? bin_of(key) : -1;
        return Put{at, W && at >= 0 ? weight_of(chance(key)) : SmWeight{0, 0}};
      }, [&](const Put& a) { put(q, a); });
      if (W && more && rank == 0 && tid == 0) put_whole(q, bin_of(more_key), more);
      find_bin<W>(s, q, before, target, 1.0, n_cta, rank);
      hi -= min(s.found_bin << bits, hi - lo);
      if (hi - lo > (1u << bits) - 1) lo = hi - ((1u << bits) - 1);
    }
    // a key whose low bits are its type's: zeros above 0, ones below
    return KS == 0 ? hi : (hi & (0x80000000u >> KS)) ? hi << KS : (hi << KS) | ((1u << KS) - 1);
  };
  if (by_k) {
    // Every warp has a key that is not below `least`: the k largest are not either.
    if (n_cta > 1 && k <= (int)n_cta * kSmWarps && least > kSmNone) {
      mark_from(least);
      if (!gather()) return;
      if (n_cta == 1) mark_from(least);
    }
    cut_key = search(std::false_type(), [](uint32_t) { return true; }, 0, 0, 0, (u64)k, 1.0, 0);
    if (gone) return;
    cut_ties = (u64)k - s.found_before;
    some_ties = cut_ties < s.found_in;
    __syncthreads();
  }
  if (by_p) {
    const uint32_t k_key = cut_key;
    const u64 k_ties = cut_ties;
    // All logits below this one together weigh less than 1 - top_p of the largest: the cut lies above. In whole units a
    // weight is at most twice what it was (below half a unit it is 0), so each has half of its share; the rest is room for roundings.
    const float tail = top + t * (logf((1.f - top_p) / (2.f * (float)a.V)) - 0.01f);
    const uint32_t tail_key = top_p > 0.f && tail - 1e-5f * fabsf(top) > -INFINITY ? min(key_of(tail - 1e-5f * fabsf(top)), most) : 0u;
    // of the equals of top-k's last, the kept ones
    const uint32_t key = search(std::true_type(), [&](uint32_t q) { return q > k_key || (q == k_key && k_ties == ~0ull); }, k_key, k_key,
                                k_ties == ~0ull ? 0 : k_ties * weight(chance(k_key)), 0, (double)top_p, tail_key);
    if (gone) return;
    const u64 one = weight(chance(key)), before = s.found_before;
    if (one > 0) {
      // the fewest equals whose weight takes the sum to the target
      const u64 n = (s.found_target - before + one - 1) / one;   // at least 1: `before` is below the target
      const u64 all = s.found_in / one;
      if (n < all || key != k_key) some_ties = n < all;
      cut_key = key;
      cut_ties = n < all ? n : all;
    }
    __syncthreads();
  }
  uint32_t last = 0xffffffffu;   // equals of cut_key are kept up to this index
  const uint32_t last_key = cut_key;
  if (some_ties) last = nth(cut_key, cut_ties);

  // ---- the draw
  const float min_p = floor_p > 0.f ? fminf(floor_p, 1.f) : 0.f;
  // keys below this weigh nothing, or less than min_p: exp(z) >= min_p asks for a z that is a little
  // below its logarithm at least, with room for the logarithm's and the other roundings
  {
    const float z = min_p > 0.f ? fmaxf(logf(min_p), -28.5f) : -28.5f;
    const float low = top + t * z - 1e-5f * (fabsf(top) + 2.f * t * fabsf(z) + t);
    if (low > -INFINITY) cut_key = max(cut_key, key_of(low));
    cut_key = min(cut_key, most);   // the first is always kept
  }
  const bool ties = last != 0xffffffffu;
  auto kept = [&](int i, uint32_t key) -> SmWeight {   // number i of the slice
    const float w = chance(key);
    bool drop = key < cut_key || w < min_p;
    if (ties && key == last_key) drop |= index_of(i) > last;
    return weight_of(drop ? 0.f : w);
  };
  SmWeight some = {0, 0};   // bits added up, and how many
  uint32_t n_some = 0;
  auto add = [&](const SmWeight& w) {
    some.a += w.a;
    some.b += w.b;
    ++n_some;
  };
  if (few()) {
    each_of(can, [&](int i, uint32_t key) { return kept(tid * chunk + i, key); }, add);
  } else {
    by_four(cut_key, [&](int i, const uint32_t (&k4)[4]) {
#pragma unroll
      for (int j = 0; j < 4; ++j) add(kept(tid * chunk + i + j, k4[j]));
    });
  }
  const u64 sum = ((u64)(some.a - n_some * 0x41000000u) << 20) + (some.b - n_some * 0x37000000u);
  u64 all;
  const u64 before = row_before(sum, s, round, &all, n_cta, rank);
  const double mark_d = (double)a.u[row] * (double)all;
  u64 mark = mark_d > 0.0 ? (u64)mark_d : 0;
  if (mark > all - 1) mark = all - 1;
  const int i = walk(before, sum, mark, [&](int i) { return kept(i, keys[i]).whole(); });
  if (i >= 0 && lane == 0) {
    a.token[row] = (int32_t)index_of(i);
    if (a.logprob) {
      const float rest = (float)((double)(all - (u64)kSmUnit) / (double)kSmUnit);
      a.logprob[row] = logit_of(keys[i]) - log1pf(rest);
    }
  }
  row_sync(n_cta);   // no CTA leaves while another reads its shared memory
}

}  // namespace

cudaError_t sample(int dtype, const Sample& a, const Dev& dev) {
  const int n_cta = a.V > 4096 ? kSmMostCluster : 1;
  int chunk = (a.V + n_cta * kSmThreads - 1) / (n_cta * kSmThreads);
  chunk |= 1;
  if (chunk > kSmMostChunk || (int64_t)a.B * n_cta > INT32_MAX) return cudaErrorInvalidValue;
  auto run = [&](auto t) -> cudaError_t {
    using T = decltype(t);
    const cudaError_t e = allow_smem<sample_kernel<T>, kSmSmem>();
    if (e != cudaSuccess) return e;
    return launch_pdl_cluster(sample_kernel<T>, dim3((unsigned)(a.B * n_cta)), dim3(kSmThreads),
                              (size_t)kSmThreads * chunk * 4 + 16, dev.stream, n_cta, a, chunk);
  };
  return dtype == kBF16 ? run(bf16()) : run(0.f);
}

}  // namespace adadsf
