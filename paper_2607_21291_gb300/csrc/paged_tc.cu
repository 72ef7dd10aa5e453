// Attention of chunks of new tokens over a paged cache on the 5th-generation tensor
// cores, bf16 (adadsf_paged_attention).
//
// A row tile is 128 TMEM lanes: R = 128 / G tokens (rounded down) times the G query heads that
// share a key/value head, so the heads of a group read its keys and values once. An item is
// two row tiles (2 R tokens) of one key/value head; they share every block of 128
// keys and take turns: while one tile's softmax runs, the tensor cores work for the
// other. Items lie on one line of blocks cut into equal pieces, one per SM (see PagedLine), so chunks
// of any mix of lengths, and few rows over a long cache, fill the machine. Pieces of a cut
// item leave fp32 partials; the one that finishes last joins them in order (many of them in two steps).
//   warp 0      TMA: Q tiles of the item; bf16 caches: K and V blocks, a box a page
//   warp 1      issues S_t = Q_t K^T (M = N = 128) into TMEM and, once the tile's softmax has
//               written P_t over S_t, O_t += P_t V: P_t from TMEM, V as it lies in the pages (an
//               MN-major operand). Order: S_0(j) S_1(j) P_0V(j) S_0(j+1) P_1V(j) S_1(j+1) ...
//   warps 2, 3  bf16 caches: V rows that not every row may see, before their product: keys past
//               the end become zeros, infinities and NaN of other new tokens are taken out
//               (zero times them is NaN) and given to the rows that see them at the end
//   warps 4-11  softmax, a tile each four warps, one row a thread: the 128 scores of a
//               block stay in registers between the maximum and the exponentials; a row maximum
//               up to 2^8 too low saves most rescaling of O
//   warps 12-15 8-bit caches: K and V numbers to bf16 in the operands' layout (read
//               a block ahead into registers); key scales multiply scores, value scales
//               weights, both through shared memory
// Weights enter the product as bf16. Where a row sees few keys their rounding does not average
// out, so items of at most kPtFine keys add a second product with what the rounding left.
// Every wait is bounded in time (device error word on give-up).
//
// Measured, 28 query heads on 4 of 128: 2048 tokens on 14336 cached 392 us, 1150 TFLOP/s (60% of a plain product's;
// about 50 us of it do not grow with the cache, the slope is 1270). The chain softmax, product, next scores of a tile
// bounds it: the tensor cores are busy 45% of the time, with only products issued they would reach 1500. 8-bit caches
// take 659 us: conversion and scales share the schedulers with the softmax (a fifth
// less without the conversion, a third less without the scales besides; scales read again instead of scaled scores written back
// were 4% slower). 7 ragged
// chunks of 777 on up to 3001 in 8 bits, 12 query heads on 2: 126 us; 128 tokens on 100: 13.6 us.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace adadsf {
namespace {

constexpr int kPtRows = 128;            // lanes of a row tile
constexpr int kPtKB = 128;              // keys of a block
constexpr int kPtMaxCtas = 160;
constexpr int kPtPad = 2;               // an item's start and end, in blocks
constexpr int kPtWhole = 4;             // blocks up to which an item is not cut
constexpr int kPtFine = 2048;           // keys up to which weights enter in two parts
constexpr int kPtJoin = 8;              // pieces that are joined at a time
constexpr int kPtGroups = 512;          // first counter of such groups
static_assert(2 * kPtMaxCtas <= kPtGroups && (kPtGroups + 4 * kPtMaxCtas) * 4 <= (int)kSyncBytes, "counters");
constexpr float kPtRescale = 8.f;       // O rescaled only when the row maximum grows by > 2^8

template <int HD, bool I8>
struct PtCfg {
  static constexpr int THREADS = I8 ? 512 : 384;
  static constexpr int KST = HD == 64 ? 4 : I8 ? 2 : 3;
  static constexpr int VST = HD == 64 ? 4 : 2;
  static constexpr int HS = HD / 64;                // 64-feature slabs
  static constexpr int SLAB = 128 * 128;            // 128 rows of 128 bytes
  static constexpr int TILE = HS * SLAB;            // Q tile, K block or V block
  // 8-bit numbers on their way: halves of a block's keys (or values), 64 rows of HD bytes as they lie
  static constexpr int GST = I8 ? (HD == 64 ? 6 : 3) : 0;
  static constexpr int GSTN = GST ? GST : 1;
  static constexpr int GHALF = 64 * HD;
  static constexpr int DATA = (2 + KST + VST) * TILE + GST * GHALF;
  // key and value scales of eight blocks: they are written up to KST blocks ahead of the one that the softmax reads
  static constexpr int SC = 8;
  static_assert(KST + 1 <= SC, "scales");
  static constexpr int SCW = 2 * kPtKB + 4;          // words of a block: keys, values, marks of keys that are NaN
  static constexpr int SCALES = I8 ? SC * SCW * 4 : 0;
  static constexpr int NBARS = 2 + 2 * KST + 3 * VST + 8 + 1 + SC + 4 + 2 * GST;
  static constexpr int TAIL = 512;
  static constexpr int RAW = DATA + SCALES + TAIL + 1024;
  static constexpr int SMEM = RAW > 232448 ? 232448 : RAW < 120 * 1024 ? 120 * 1024 : RAW;   // one CTA an SM: TMEM is allocated in full
  static constexpr int SLACK = SMEM - DATA - SCALES - TAIL;
  static_assert(SLACK >= 256 && NBARS * 8 + 64 <= TAIL, "shared memory");
  // TMEM columns: S_0 (P_0 over it) at 0, S_1 at 128, O_0 at 256, O_1 at 256 + HD
  static constexpr uint32_t TO = 256;
  static constexpr int PART = 2 * (kPtRows * HD + 2 * kPtRows) + 64;   // floats of a piece: per tile O, (m, l); then flags
};

// Groups of two row tiles, blocks of 128 keys.
struct PtCut {
  static constexpr int KEYS = kPtKB, PAD = kPtPad, WHOLE = kPtWhole;
  int R;
  __device__ __forceinline__ int groups(int n) const { return (n + 2 * R - 1) / (2 * R); }
  __device__ __forceinline__ int tokens(int g) const { return (g + 1) * 2 * R; }
};

// A piece of an item on a CTA: blocks j0 .. j1 - 1; nb[t]: blocks that tile t takes in all.
struct PtWork {
  PagedItem<PtCut> it;
  int j0, j1, two, nb[2];
  int t0;      // first token
  bool mine;   // whether the piece has the item's start
  __device__ __forceinline__ int open(int t, int R) const { return it.len - it.n + t0 + t * R + 1; }   // keys that its first row sees
};
__device__ __forceinline__ PtWork pt_work(const PagedItem<PtCut>& it, int64_t ua, int64_t ub, int R) {
  PtWork w;
  w.it = it;
  w.t0 = it.grp * 2 * R;
  w.two = it.n > w.t0 + R;
  const int seen0 = max(0, it.len - it.n + min(it.n, w.t0 + R));
  w.nb[0] = (seen0 + kPtKB - 1) / kPtKB;
  w.nb[1] = w.two ? (it.seen + kPtKB - 1) / kPtKB : 0;
  it.in(ua, ub, &w.j0, &w.j1);
  w.mine = w.j0 == 0 && w.j1 > 0;
  w.j1 = min(w.j1, w.two ? w.nb[1] : w.nb[0]);
  return w;
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* tmap, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}
// Shared-memory descriptors as a word that holds the address (in 16 bytes) and one that does not. Q and K
// (K-major): rows of 128 bytes, groups of eight 1024 apart. V as it lies (MN-major): 64
// features (128 bytes) a row, keys as rows, the next eight keys 1024 bytes on, the next 64 features `slab`.
constexpr uint32_t kDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr, uint32_t slab) { return ((saddr & 0x3FFFFu) >> 4) | (slab >> 4) << 16; }
// The products of a warp whose lanes all come here, issued by the one with lead != 0: with
// warp-uniform operands they need no moves between register files (a single lane in a branch
// of its own took 100 clocks a product).
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %6};\n\tmov.b64 db, {%2, %6};\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(lead), "r"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b, uint32_t idesc, uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %6};\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
      "r"(a_tmem), "r"(b), "r"(idesc), "r"(acc), "r"(lead), "r"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(lead)
      : "memory");
}
template <int HD, bool I8>
__global__ void __launch_bounds__(PtCfg<HD, I8>::THREADS, 1)
    paged_tc_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                    const __grid_constant__ CUtensorMap tv, const Paged p, bf16* out, float scale_log2, int* sync,
                    float* parts, int* err, unsigned long long timeout_ns) {
  using C = PtCfg<HD, I8>;
  constexpr int KST = C::KST, VST = C::VST;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  if (smem - smem_raw > C::SLACK) {   // the layout would not fit: report and touch nothing
    if (threadIdx.x == 0) set_device_error(err, DEVERR_TIMEOUT);
    return;
  }
  const uint32_t sQ = smem_u32(smem), sK0 = sQ + 2 * C::TILE, sV0 = sK0 + KST * C::TILE, sG0 = sV0 + VST * C::TILE;
  float* scales = reinterpret_cast<float*>(smem + C::DATA);           // [SC][SCW]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::DATA + C::SCALES);
  const uint32_t q_full = smem_u32(bars), q_empty = q_full + 8;
  const uint32_t k_full0 = q_empty + 8, k_empty0 = k_full0 + 8 * KST;
  const uint32_t v_full0 = k_empty0 + 8 * KST, v_empty0 = v_full0 + 8 * VST, v_ok0 = v_empty0 + 8 * VST;
  const uint32_t s_full0 = v_ok0 + 8 * VST, p_full0 = s_full0 + 16, o_done0 = p_full0 + 16, o_free0 = o_done0 + 16;
  const uint32_t drain = o_free0 + 16, sc_full0 = drain + 8, wrote0 = sc_full0 + 8 * C::SC, told0 = wrote0 + 16;
  const uint32_t g_full0 = told0 + 16, g_empty0 = g_full0 + 8 * C::GST;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NBARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* last_s = abort_flag + 1;      // [2] whether this CTA joins the tile's pieces
  int* odd_s = const_cast<int*>(last_s) + 2;  // pieces whose V held an infinity or NaN that was taken out

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = p.Hq / p.Hkv, R = kPtRows / G;
  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int i = 0; i < KST; ++i) {
      mbar_init(k_full0 + 8 * i, I8 ? 4 : 1);
      mbar_init(k_empty0 + 8 * i, 1);
    }
    for (int i = 0; i < VST; ++i) {
      mbar_init(v_full0 + 8 * i, I8 ? 4 : 1);
      mbar_init(v_empty0 + 8 * i, 1);
      mbar_init(v_ok0 + 8 * i, 2);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full0 + 8 * t, 1);
      mbar_init(p_full0 + 8 * t, 4);
      mbar_init(o_done0 + 8 * t, 1);
      mbar_init(o_free0 + 8 * t, 4);
    }
    mbar_init(drain, 1);
    for (int i = 0; i < C::SC; ++i) mbar_init(sc_full0 + 8 * i, 4);
    for (int i = 0; i < C::GST; ++i) {
      mbar_init(g_full0 + 8 * i, 1);
      mbar_init(g_empty0 + 8 * i, 4);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(wrote0 + 8 * t, 4);
      mbar_init(told0 + 8 * t, 1);
    }
    *abort_flag = 0;
    *odd_s = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tq);
    tma_prefetch_desc(&tk);
    tma_prefetch_desc(&tv);
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), 512);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();

  PagedLine<PtCut> line{PtCut{R}};
  int64_t per, ua, ub;
  line.piece(p, kPtPad + 1, (int)blockIdx.x, (int)gridDim.x, lane, err, &per, &ua, &ub);
  auto wait = [&](uint32_t bar, uint32_t parity) { return paged_wait(bar, parity, abort_flag, err, timeout_ns); };
  auto all_wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
  // a lane waits for its warp
  auto warp_wait = [&](uint32_t bar, uint32_t parity) {
    int w = 0;
    if (lane == 0) w = wait(bar, parity);
    return __shfl_sync(0xffffffffu, w, 0) != 0;
  };

  if (warp < 4) {
    if (warp == 0) {
      // ------------------------------------------------------------ TMA
      const int box = I8 ? min(1 << p.page_log2, 64) : 1 << p.page_log2, boxes = kPtKB / box;   // rows of a copy, copies of a block
      int items = 0, issued = 0, copied = 0;
      bool ok = true;
      for (int64_t u = ua; ok && u < ub;) {
        const PagedItem<PtCut> it = line.item(p, &u, lane, err);
        const PtWork w = pt_work(it, ua, ub, R);
        if (w.j0 >= w.j1) continue;
        if (items > 0 && !warp_wait(q_empty, (items - 1) & 1)) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(q_full, (uint32_t)((w.two ? 2 : 1) * C::HS * R * G * 128));
          for (int t = 0; t < (w.two ? 2 : 1); ++t)
            for (int s = 0; s < C::HS; ++s)
              tma_load_4d(sQ + t * C::TILE + s * C::SLAB, &tq, s * 64, 0, it.h, (int)(it.row0 + w.t0 + t * R), q_full);
        }
        ++items;
        const int32_t* tab = p.table + (int64_t)it.b * p.max_pages;
        auto page_of = [&](int j) {
          const int place = j * kPtKB + lane * box;
          return lane < boxes && place < it.seen ? tab[place >> p.page_log2] : 0;
        };
        int next = page_of(w.j0);
        for (int j = w.j0; j < w.j1; ++j) {
          const int page = next;
          if (j + 1 < w.j1) next = page_of(j + 1);
          const int place = j * kPtKB + lane * box;
          const bool want = lane < boxes && place < it.seen;
          const bool there = (unsigned)page < (unsigned)p.n_pages;
          if (want && !there) set_device_error(err, DEVERR_INDEX);
          const int z = there ? page * p.Hkv + it.h : p.n_pages * p.Hkv;   // out of the pool: filled with zeros
          const unsigned wants = __ballot_sync(0xffffffffu, want);
          const int r = place & ((1 << p.page_log2) - 1);
          if (I8) {
            // keys, then values, in halves: half h is the copies of lanes boxes / 2 h ..
            const int half = boxes / 2, mine = lane >= half, at = lane - mine * half;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int st = copied % C::GSTN;
              const unsigned part = (v & 1) ? wants >> half : wants & ((1u << half) - 1);
              ok = ok && all_wait(g_empty0 + 8 * st, ((copied / C::GSTN) & 1) ^ 1);
              if (!ok) break;
              if (lane == 0) mbar_arrive_expect_tx(g_full0 + 8 * st, (uint32_t)(__popc(part) * box * HD));
              __syncwarp();
              if (want && mine == (v & 1)) tma_load_3d(sG0 + st * C::GHALF + at * box * HD, v < 2 ? &tk : &tv, 0, r, z, g_full0 + 8 * st);
              ++copied;
            }
            if (!ok) break;
            continue;
          }
          const uint32_t bytes = (uint32_t)(__popc(wants) * box * C::HS * 128);
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const int n_st = v ? VST : KST, st = issued % n_st;
            const uint32_t full = (v ? v_full0 : k_full0) + 8 * st, empty = (v ? v_empty0 : k_empty0) + 8 * st;
            if (!all_wait(empty, ((issued / n_st) & 1) ^ 1)) { ok = false; break; }
            if (lane == 0) mbar_arrive_expect_tx(full, bytes);
            __syncwarp();
            if (want)
#pragma unroll
              for (int s = 0; s < C::HS; ++s)
                tma_load_3d((v ? sV0 : sK0) + st * C::TILE + s * C::SLAB + lane * box * 128, v ? &tv : &tk, s * 64, 0, z, full);
          }
          if (!ok) break;
          ++issued;
        }
      }
      pdl_trigger();
      // drain: what was copied last into each place has landed
      if (lane == 0) {
        if (items > 0) mbar_wait_drain(q_full, (items - 1) & 1, timeout_ns);
        if (I8)
          for (int st = 0; st < C::GST && st < copied; ++st) {
            const int last = st + ((copied - 1 - st) / C::GSTN) * C::GSTN;
            mbar_wait_drain(g_full0 + 8 * st, (uint32_t)((last / C::GSTN) & 1), timeout_ns);
          }
        else
          for (int v = 0; v < 2; ++v) {
            const int n_st = v ? VST : KST;
            for (int st = 0; st < n_st && st < issued; ++st) {
              const int last = st + ((issued - 1 - st) / n_st) * n_st;
              mbar_wait_drain((v ? v_full0 : k_full0) + 8 * st, (uint32_t)((last / n_st) & 1), timeout_ns);
            }
          }
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------ products
      constexpr uint32_t idesc_s = idesc_bf16_f32(kPtRows, kPtKB);
      constexpr uint32_t idesc_o = idesc_bf16_f32(kPtRows, HD) | (1u << 16);   // B is MN-major
      const uint32_t lead = lane == 0;
      const uint32_t q_low = desc_low(sQ, 0), k_low = desc_low(sK0, 0), v_low = desc_low(sV0, C::SLAB);
      auto issue_s = [&](int t, int kslot) {
        const uint32_t q0 = q_low + t * (C::TILE >> 4), k0 = k_low + kslot * (C::TILE >> 4), d = tmem_base + t * kPtKB;
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * C::SLAB + (kk & 3) * 32) >> 4;
          mma_ss(d, q0 + off, k0 + off, idesc_s, kk > 0 ? 1u : 0u, lead);
        }
        commit(s_full0 + 8 * t, lead);
      };
      auto issue_pv = [&](int t, int vslot, bool acc, bool fine) {
        const uint32_t v0 = v_low + vslot * (C::TILE >> 4), to = tmem_base + C::TO + t * HD, tp = tmem_base + t * kPtKB;
#pragma unroll
        for (int kk = 0; kk < kPtKB / 16; ++kk)
          mma_ts(to, tp + (kk >> 1) * 32 + (kk & 1) * 8, v0 + kk * 128, idesc_o, (acc || kk > 0) ? 1u : 0u, lead);
        if (fine)
#pragma unroll
          for (int kk = 0; kk < kPtKB / 16; ++kk) mma_ts(to, tp + (kk >> 1) * 32 + 16 + (kk & 1) * 8, v0 + kk * 128, idesc_o, 1u, lead);
        commit(o_done0 + 8 * t, lead);
      };
      int kc = 0, vc = 0, items = 0;
      int pc[2] = {0, 0}, oc[2] = {0, 0};   // P blocks taken, pieces finished, per tile
      bool ok = true;
      for (int64_t u = ua; ok && u < ub;) {
        const PagedItem<PtCut> it = line.item(p, &u, lane, err);
        const PtWork w = pt_work(it, ua, ub, R);
        if (w.j0 >= w.j1) continue;
        const bool fine = it.seen <= kPtFine;
        auto k_wait = [&](int c) { return all_wait(k_full0 + 8 * (c % KST), (c / KST) & 1); };
        ok = all_wait(q_full, items & 1) && k_wait(kc);
        if (!ok) break;
        tc_fence_after();
        // S_t may overwrite the last piece's P_t: its product was issued before
        if (w.j0 < w.nb[0]) issue_s(0, kc % KST);
        if (w.two) issue_s(1, kc % KST);
        commit(k_empty0 + 8 * (kc % KST), lead);
        for (int j = w.j0; j < w.j1; ++j) {
          const bool next = j + 1 < w.j1;
          const int vslot = vc % VST, knext = (kc + 1) % KST;
          // bf16: V that some row may not see has been looked at
          if (!I8) ok = all_wait(v_ok0 + 8 * vslot, (vc / VST) & 1);
          ok = ok && all_wait(v_full0 + 8 * vslot, (vc / VST) & 1);
          if (!ok) break;
          if (j < w.nb[0]) {
            ok = all_wait(p_full0, pc[0] & 1);
            ++pc[0];
            // the first product of a piece overwrites O_0: the last piece's must have been read
            if (j == w.j0 && oc[0] > 0) ok = ok && all_wait(o_free0, (oc[0] - 1) & 1);
            if (!ok) break;
            tc_fence_after();
            issue_pv(0, vslot, j > w.j0, fine);
          }
          if (next && !k_wait(kc + 1)) { ok = false; break; }
          tc_fence_after();
          if (next && j + 1 < w.nb[0]) issue_s(0, knext);
          if (w.two) {
            ok = all_wait(p_full0 + 8, pc[1] & 1);
            ++pc[1];
            if (j == w.j0 && oc[1] > 0) ok = ok && all_wait(o_free0 + 8, (oc[1] - 1) & 1);
            if (!ok) break;
            tc_fence_after();
            issue_pv(1, vslot, j > w.j0, fine);
            if (next) issue_s(1, knext);
          }
          commit(v_empty0 + 8 * vslot, lead);
          ++vc;
          if (next) {
            commit(k_empty0 + 8 * knext, lead);
            ++kc;
          }
        }
        ++kc;
        if (w.j0 < w.nb[0]) ++oc[0];
        if (w.two) ++oc[1];
        if (ok) commit(q_empty, lead);
        ++items;
      }
      __syncwarp();
      if (lane == 0) {
        tc_commit(drain);
        mbar_wait_drain(drain, 0, timeout_ns);
      }
      __syncwarp();
    } else if (!I8) {
      // ------------------------------------------------------------ V of keys that not every row sees
      int vc = 0;
      bool ok = true;
      for (int64_t u = ua; ok && u < ub;) {
        const PagedItem<PtCut> it = line.item(p, &u, lane, err);
        const PtWork w = pt_work(it, ua, ub, R);
        const int open = w.open(0, R);
        for (int j = w.j0; j < w.j1; ++j, ++vc) {
          const int st = vc % VST;
          if (!warp_wait(v_full0 + 8 * st, (vc / VST) & 1)) { ok = false; break; }
          if ((j + 1) * kPtKB > open) {
            // rows of 128 bytes, eight lanes each; this warp every other four
            const int k0 = max(open, j * kPtKB) - j * kPtKB;
            int odd = 0;
            for (int r = (k0 & ~7) + (warp & 1) * 4 + (lane >> 3); r < kPtKB; r += 8) {
              if (r < k0) continue;
#pragma unroll
              for (int s = 0; s < C::HS; ++s) {
                uint4* a = reinterpret_cast<uint4*>(smem + (sV0 - sQ) + st * C::TILE + s * C::SLAB + r * 128 + (lane & 7) * 16);
                if (j * kPtKB + r >= it.seen) {
                  *a = make_uint4(0, 0, 0, 0);
                  continue;
                }
                const uint4 x = *a;
                uint32_t y[4] = {x.x, x.y, x.z, x.w};
                bool bad = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  if ((y[i] & 0x7f80u) == 0x7f80u) { y[i] &= 0xffff0000u; bad = true; }
                  if ((y[i] & 0x7f800000u) == 0x7f800000u) { y[i] &= 0xffffu; bad = true; }
                }
                if (bad) {
                  *a = make_uint4(y[0], y[1], y[2], y[3]);
                  odd = 1;
                }
              }
            }
            if (odd) atomicOr(odd_s, 1);
            fence_proxy_async_smem();   // written by threads, read by the product
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(v_ok0 + 8 * st);
        }
      }
    }
  } else if (warp < 12) {
    // -------------------------------------------------------------- softmax

    const int t = (warp - 4) >> 2;                   // tile
    const int r = (warp & 3) * 32 + lane;            // its row = TMEM lane
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem_base + t * kPtKB + lane_off, tO = tmem_base + C::TO + t * HD + lane_off;
    const int ti = r / G;                            // its token in the tile (R and more: none)
    const int gi = r - ti * G;
    int sc = 0, blocks = 0, cut = 0;   // S blocks taken, blocks passed, pieces of cut items
    bool ok = true;
    for (int64_t u = ua; ok && u < ub;) {
      const PagedItem<PtCut> it = line.item(p, &u, lane, err);
      const PtWork w = pt_work(it, ua, ub, R);
      const int i = w.t0 + t * R + ti;
      const bool live = ti < R && i < it.n;
      const int lim = live ? it.len - it.n + i + 1 : 0;   // keys that the row sees
      bf16* dst = out + ((it.row0 + i) * p.Hq + it.h * G + gi) * HD;
      const int j1 = min(w.j1, w.nb[t]);
      if (w.nb[t] == 0 && w.mine && live && (t == 0 || w.two))   // a tile without keys
        for (int e = 0; e < HD; e += 8) *reinterpret_cast<uint4*>(dst + e) = make_uint4(0, 0, 0, 0);
      if (w.j0 >= j1) {
        blocks += max(0, w.j1 - w.j0);
        continue;
      }
      const bool fine = it.seen <= kPtFine;
      const int open = w.open(t, R);
      float m = -INFINITY, l = 0.f;
      for (int j = w.j0; j < j1; ++j) {
        const int at_sc = (blocks + j - w.j0) % C::SC;
        const float4* ks4 = reinterpret_cast<const float4*>(scales + at_sc * C::SCW);
        const float4* vs4 = ks4 + kPtKB / 4;
        if (I8 && !all_wait(sc_full0 + 8 * at_sc, (blocks + j - w.j0) / C::SC & 1)) { ok = false; break; }
        if (!all_wait(s_full0 + 8 * t, sc & 1)) { ok = false; break; }
        ++sc;
        tc_fence_after();
        const uint4 marks = I8 ? reinterpret_cast<const uint4*>(vs4)[kPtKB / 4] : make_uint4(0, 0, 0, 0);
        if ((j + 1) * kPtKB > open || (marks.x | marks.y | marks.z | marks.w)) {
          // keys that the row does not see: -infinity
          const int left = lim - j * kPtKB;
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            uint32_t z[32];
            tmem_ld32(tS + 32 * c, z);
            tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              if (I8 && ((c == 0 ? marks.x : c == 1 ? marks.y : c == 2 ? marks.z : marks.w) >> k & 1)) z[k] = 0x7fc00000u;
              z[k] = 32 * c + k < left ? z[k] : 0xff800000u;
            }
            tmem_st32(tS + 32 * c, z);
          }
          tmem_st_wait();
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        constexpr int MW = I8 ? 32 : 64;   // scores read at once
#pragma unroll 1
        for (int c = 0; c < kPtKB; c += MW) {
          uint32_t s[MW];
#pragma unroll
          for (int i = 0; i < MW; i += 32) tmem_ld32(tS + c + i, s + i);
          tmem_ld_wait();
#pragma unroll
          for (int k = 0; k < MW; k += 4) {
            float4 y = make_float4(__uint_as_float(s[k]), __uint_as_float(s[k + 1]), __uint_as_float(s[k + 2]), __uint_as_float(s[k + 3]));
            if (I8) {   // the scale of the scores is in the key scales
              const float4 f = ks4[(c + k) / 4];
              const float2 u0 = __fmul2_rn(make_float2(y.x, y.y), make_float2(f.x, f.y));
              const float2 u1 = __fmul2_rn(make_float2(y.z, y.w), make_float2(f.z, f.w));
              y = make_float4(u0.x, u0.y, u1.x, u1.y);
            }
            mx[(k >> 1) & 3] = fmax3(mx[(k >> 1) & 3], y.x, y.y);
            mx[((k >> 1) + 1) & 3] = fmax3(mx[((k >> 1) + 1) & 3], y.z, y.w);
            if (I8) {
              s[k] = __float_as_uint(y.x); s[k + 1] = __float_as_uint(y.y);
              s[k + 2] = __float_as_uint(y.z); s[k + 3] = __float_as_uint(y.w);
            }
          }
          if (I8) tmem_st32(tS + c, s);
        }
        if (I8) tmem_st_wait();
        float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        if (!I8) top *= scale_log2;
        // O is stable: its last product was issued before S_t(j), which is complete
        const bool grow = top > m + kPtRescale;          // true for the first finite maximum
        if (__any_sync(0xffffffffu, grow && m > -INFINITY)) {
          const float alpha = grow ? (m > -INFINITY ? ex2_approx(m - top) : 1.f) : 1.f;
          l *= alpha;
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t o[32];
            tmem_ld32(tO + c * 32, o);
            tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
            tmem_st32(tO + c * 32, o);
          }
        }
        if (grow) m = top;
        const float base = m == -INFINITY ? 0.f : m;
        const float2 scale2 = make_float2(scale_log2, scale_log2), neg2 = make_float2(-base, -base);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        // weights of 32 keys from their scores, over them: bf16 pairs, then what the rounding leaves
        auto weigh = [&](int c, const uint32_t (&z)[32]) {
          uint32_t hi[16];
          float2 e[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float2 y = make_float2(__uint_as_float(z[2 * k]), __uint_as_float(z[2 * k + 1]));
            y = I8 ? __fadd2_rn(y, neg2) : __ffma2_rn(y, scale2, neg2);
            e[k] = make_float2(ex2_approx(y.x), ex2_approx(y.y));
            sum[k & 1] = __fadd2_rn(sum[k & 1], e[k]);
            if (I8) {
              const float4 f = vs4[8 * c + k / 2];
              e[k] = __fmul2_rn(e[k], (k & 1) ? make_float2(f.z, f.w) : make_float2(f.x, f.y));
            }
            hi[k] = pack_bf16x2(e[k].x, e[k].y);
          }
          tmem_st16(tS + 32 * c, hi);
          if (fine) {
#pragma unroll
            for (int k = 0; k < 16; ++k)
              hi[k] = pack_bf16x2(e[k].x - __uint_as_float(hi[k] << 16), e[k].y - __uint_as_float(hi[k] & 0xffff0000u));
            tmem_st16(tS + 32 * c + 16, hi);
          }
        };
        // read again piece by piece: the loop is short enough for the instruction caches
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t z[32];
          tmem_ld32(tS + 32 * c, z);
          tmem_ld_wait();
          weigh(c, z);
        }
        l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full0 + 8 * t);
      }
      if (!ok) break;
      blocks += w.j1 - w.j0;
      if (!warp_wait(o_done0 + 8 * t, (sc - 1) & 1)) { ok = false; break; }
      tc_fence_after();
      // ---- the piece's result: out, or a partial
      const int first = it.first_cta(per), last = it.last_cta(per, w.nb[t] - 1);
      auto part_of = [&](int cta) {   // this tile's O [HD / 4][128] float4, then (m, l)
        return parts + ((int64_t)cta * 2 + (cta == first ? 1 : 0)) * C::PART + t * (kPtRows * HD + 2 * kPtRows);
      };
      auto flag_of = [&](int cta) {
        return reinterpret_cast<int*>(parts + ((int64_t)cta * 2 + (cta == first ? 1 : 0)) * C::PART + 2 * (kPtRows * HD + 2 * kPtRows)) + t;
      };
      int odd = *(volatile int*)odd_s;   // set by this item's V or an earlier one's: a look too many costs time only
      bool join = false;
      if (first != last) {
        float4* po = reinterpret_cast<float4*>(part_of((int)blockIdx.x));
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t o[32];
          tmem_ld32(tO + c * 32, o);
          tmem_ld_wait();
#pragma unroll
          for (int k = 0; k < 8; ++k)
            __stcg(po + (c * 8 + k) * kPtRows + r, make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]),
                                                               __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3])));
        }
        __stcg(reinterpret_cast<float2*>(part_of((int)blockIdx.x) + kPtRows * HD) + r, make_float2(m, l));
        if (r == 0) __stcg(flag_of((int)blockIdx.x), odd);
      }
      if (first == last) {
        const float inv = 1.f / l;
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t o[32];
          tmem_ld32(tO + c * 32, o);
          tmem_ld_wait();
          if (live) {
            float v[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = lim > 0 ? __uint_as_float(o[k]) * inv : 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) store_vec(dst + c * 32 + 8 * k, v + 8 * k);
          }
        }
      }
      // O_t is read: the next piece's first product may overwrite it
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_free0 + 8 * t);
      if (first != last) {
        // Whether this is the last of n CTAs that come here for the tile; all of the tile's threads.
        auto finish = [&](int* counter, int n) {
          __threadfence();
          __syncwarp();
          if (lane == 0) mbar_arrive(wrote0 + 8 * t);
          if (r < 32) {   // the tile's first warp counts
            if (!warp_wait(wrote0 + 8 * t, cut & 1)) return ok = false;
            if (lane == 0) {
              __threadfence();
              const int done = atomicAdd(counter, 1) == n - 1;
              if (done) *counter = 0;
              last_s[t] = done;
              __threadfence();
              mbar_arrive(told0 + 8 * t);
            }
          }
          if (!warp_wait(told0 + 8 * t, cut & 1)) return ok = false;
          ++cut;
          return last_s[t] != 0;
        };
        // Partials of CTAs from, from + step, .. to, in this order, into the first one's place, or divided by their sum into the output.
        auto merge = [&](int from, int step, int to, bool out) {
          __threadfence();
          float mm = -INFINITY, ll = 0.f;
          for (int c = from; c <= to; c += step) {
            mm = fmaxf(mm, __ldcg(reinterpret_cast<const float2*>(part_of(c) + kPtRows * HD) + r).x);
            odd |= __ldcg(flag_of(c));
          }
          const float base = mm == -INFINITY ? 0.f : mm;
          for (int c = from; c <= to; c += step) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(part_of(c) + kPtRows * HD) + r);
            ll += ml.y * ex2_approx(ml.x - base);
          }
          const float by = out ? 1.f / ll : 1.f;
          if (live) {
#pragma unroll 1
            for (int e = 0; e < HD; e += 32) {
              float v[32];
#pragma unroll
              for (int k = 0; k < 32; ++k) v[k] = 0.f;
#pragma unroll(I8 ? 1 : 2)
              for (int c = from; c <= to; c += step) {
                const float* po = part_of(c);
                const float f = ex2_approx(__ldcg(reinterpret_cast<const float2*>(po + kPtRows * HD) + r).x - base) * by;
                float4 x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = __ldcg(reinterpret_cast<const float4*>(po) + (e / 4 + k) * kPtRows + r);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  v[4 * k] = fmaf(x[k].x, f, v[4 * k]);
                  v[4 * k + 1] = fmaf(x[k].y, f, v[4 * k + 1]);
                  v[4 * k + 2] = fmaf(x[k].z, f, v[4 * k + 2]);
                  v[4 * k + 3] = fmaf(x[k].w, f, v[4 * k + 3]);
                }
              }
              if (out) {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] = lim > 0 ? v[k] : 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) store_vec(dst + e + 8 * k, v + 8 * k);
              } else {
                float4* po = reinterpret_cast<float4*>(part_of(from));
#pragma unroll
                for (int k = 0; k < 8; ++k)
                  __stcg(po + (e / 4 + k) * kPtRows + r, make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]));
              }
            }
          }
          if (!out) {
            __stcg(reinterpret_cast<float2*>(part_of(from) + kPtRows * HD) + r, make_float2(mm, ll));
            if (r == 0) __stcg(flag_of(from), odd);
          }
        };
        // Many pieces: by kPtJoin first, then these. One CTA reads 64 KB a tile and piece, 1.7 us: 12 tokens on 20000 cached of 28
        // heads on 4, in 38 pieces a head, took 73 us in one step, 48 in two; 13 pieces are faster in one.
        const int me = (int)blockIdx.x, pieces = last - first + 1;
        const int step = pieces > 2 * kPtJoin ? kPtJoin : 1;
        bool on = true;
        if (step > 1) {
          const int lead = first + (me - first) / kPtJoin * kPtJoin, end = min(lead + kPtJoin - 1, last);
          on = finish(sync + kPtGroups + (2 * lead + (lead == first)) * 2 + t, end - lead + 1);
          if (on && end > lead) merge(lead, 1, end, false);
        }
        if (on) join = finish(sync + 2 * first + t, (pieces + step - 1) / step);
        if (!ok) break;
        if (join) merge(first, step, last, true);
      }
      if (odd && live && (first == last || join)) {
        // infinities and NaN among the values of the item's own new tokens: to the rows that see them
#pragma unroll 1
        for (int j = max(w.open(0, R), 0); j < lim; ++j) {
          const int page = p.table[(int64_t)it.b * p.max_pages + (j >> p.page_log2)];
          if ((unsigned)page >= (unsigned)p.n_pages) continue;
          const int64_t vec = paged_vec(p, page, j, it.h);
          if (I8 && p.vs[vec] < INFINITY) continue;
#pragma unroll 1
          for (int e = 0; e < HD; ++e) {
            const float x = I8 ? NAN : __bfloat162float(static_cast<const bf16*>(p.v)[vec * HD + e]);
            if (!(fabsf(x) < INFINITY)) dst[e] = __float2bfloat16_rn(__bfloat162float(dst[e]) + x);
          }
        }
      }
    }
  } else if (I8) {
    // -------------------------------------------------------------- 8-bit blocks to bf16
    // A lane takes 16 bytes of a key at a time and stores 32. Eight lanes of a load or a store phase have
    // four neighbouring chunks of two keys r and r ^ 5, which in either swizzle hit all banks.
    constexpr int CH = HD / 16;                       // 16-byte chunks of a key
    constexpr int STEPS = 16 * CH / 32;               // a warp's 16 keys of a half: 4 or 2
    const int cw = warp - 12;
    const int chunk = HD == 128 ? (lane & 3) + 4 * (lane >> 4) : lane & 3;
    const int sub = lane >> 2;                        // hd 64: eight keys at once; hd 128: four
    int blocks = 0, taken = 0;
    bool ok = true;
    for (int64_t u = ua; ok && u < ub;) {
      const PagedItem<PtCut> it = line.item(p, &u, lane, err);
      const PtWork w = pt_work(it, ua, ub, R);
      if (w.j0 >= w.j1) continue;
      const int32_t* tab = p.table + (int64_t)it.b * p.max_pages;
      const int open = w.open(0, R);
      const int id = cw * 32 + lane;   // the key whose scales this thread brings
      // its vector in block j, or -1
      auto vec_of = [&](int j) -> int64_t {
        const int place = j * kPtKB + id;
        if (place >= it.seen) return -1;
        const int page = tab[place >> p.page_log2];
        return (unsigned)page < (unsigned)p.n_pages ? paged_vec(p, page, place, it.h) : -1;
      };
      // half a block to bf16: 64 keys from key 64 h on of a tile; keys past the last visible one: values
      // of any finite kind will do (their weights are zero), and what lies there was loaded as numbers
      auto turn = [&](uint32_t tile, int h) {
        const int st = taken % C::GSTN;
        if (!all_wait(g_full0 + 8 * st, (taken / C::GSTN) & 1)) return false;
        const uint8_t* from = smem + (sG0 - sQ) + st * C::GHALF;
        uint8_t* to = smem + (tile - sQ) + (chunk >> 2) * C::SLAB;
        const int c = (2 * chunk) & 7;
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
          const int low = HD == 128 ? (2 * (k & 1) + ((sub >> 1) & 1)) ^ ((sub & 1) * 5) : ((sub >> 1) & 3) ^ ((sub & 1) * 5);
          const int key = cw * 16 + (HD == 128 ? k >> 1 : k) * 8 + low;
          const uint4 x = HD == 128 ? *reinterpret_cast<const uint4*>(from + key * 128 + ((chunk ^ (key & 7)) << 4))
                                    : *reinterpret_cast<const uint4*>(from + key * 64 + ((chunk ^ ((key >> 1) & 3)) << 4));
          const uint32_t in[4] = {x.x, x.y, x.z, x.w};
          uint32_t y[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[2 * i] = bf16_of_i8(__byte_perm(in[i], 0, 0x4140));
            y[2 * i + 1] = bf16_of_i8(__byte_perm(in[i], 0, 0x4342));
          }
          uint8_t* row = to + (h * 64 + key) * 128;
          *reinterpret_cast<uint4*>(row + ((c ^ (key & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<uint4*>(row + (((c + 1) ^ (key & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(g_empty0 + 8 * st);
        ++taken;
        return true;
      };
      int64_t vec = vec_of(w.j0), vec_next = w.j0 + 1 < w.j1 ? vec_of(w.j0 + 1) : -1;
      float ksc = vec >= 0 ? __ldg(p.ks + vec) : 0.f, vsc = vec >= 0 ? __ldg(p.vs + vec) : 0.f;
#pragma unroll 1
      for (int j = w.j0; j < w.j1; ++j, ++blocks) {
        const int kst = blocks % KST, vst = blocks % VST;
        if (!all_wait(k_empty0 + 8 * kst, ((blocks / KST) & 1) ^ 1)) { ok = false; break; }
        // A masked score is -infinity before its scale, which therefore is a positive number: any
        // for a key of zeros, and for one whose scale is NaN (it held an infinity or a NaN), which
        // is marked. Such a value, where not every row sees it, is taken out and given to the rows that
        // see it at the end.
        const bool bad_k = !(ksc < INFINITY), bad_v = !(vsc < INFINITY) && j * kPtKB + id >= open;
        if (bad_v) atomicOr(odd_s, 1);
        float* sc = scales + blocks % C::SC * C::SCW;
        sc[id] = bad_k || ksc == 0.f ? scale_log2 : ksc * scale_log2;
        sc[kPtKB + id] = bad_v ? 0.f : vsc;
        const unsigned marks = __ballot_sync(0xffffffffu, bad_k);
        if (lane == 0) reinterpret_cast<uint32_t*>(sc + 2 * kPtKB)[cw] = marks;
        // the next block's scales, its page asked for a block ahead of them
        vec = vec_next;
        vec_next = j + 2 < w.j1 ? vec_of(j + 2) : -1;
        ksc = vec >= 0 ? __ldg(p.ks + vec) : 0.f;
        vsc = vec >= 0 ? __ldg(p.vs + vec) : 0.f;
        // keys, then values: one copy of the code for both and their halves
#pragma unroll 1
        for (int v = 0; v < 4; ++v) {
          if (v == 2) ok = all_wait(v_empty0 + 8 * vst, ((blocks / VST) & 1) ^ 1);
          ok = ok && turn(v < 2 ? sK0 + kst * C::TILE : sV0 + vst * C::TILE, v & 1);
          if (!ok) break;
          if (v & 1) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              if (v == 1) mbar_arrive(sc_full0 + 8 * (blocks % C::SC));
              mbar_arrive(v == 1 ? k_full0 + 8 * kst : v_full0 + 8 * vst);
            }
          }
        }
        if (!ok) break;
      }
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <int HD, bool I8>
cudaError_t launch_tc(const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch, const Dev& dev) {
  using C = PtCfg<HD, I8>;
  const cudaError_t e = allow_smem<paged_tc_kernel<HD, I8>, C::SMEM>();
  if (e != cudaSuccess) return e;
  const int G = p.Hq / p.Hkv, R = kPtRows / G;
  CUtensorMap tq, tk, tv;
  if (!make_tmap_heads(&tq, q, p, ld_q, R)) return cudaErrorInvalidValue;
  const uint32_t box = I8 ? kPtKB / 2 : kPtKB;
  if (!make_tmap_pages(&tk, p.k, p, I8, box) || !make_tmap_pages(&tv, p.v, p, I8, box)) return cudaErrorInvalidValue;
  // no more CTAs than pieces of the least size that any counts could make
  const int64_t span = ((int64_t)p.max_pages << p.page_log2) / kPtKB + 1;
  const int64_t groups = std::min<int64_t>(p.B * (((int64_t)p.max_new + 2 * R - 1) / (2 * R)), p.n_rows);
  const int64_t most = std::max<int64_t>(1, (groups * p.Hkv * (span + kPtPad) + kPtPad) / (kPtPad + 1));
  return launch_pdl(paged_tc_kernel<HD, I8>, dim3((unsigned)std::min<int64_t>(most, std::min(dev.num_sms, kPtMaxCtas))),
                    dim3(C::THREADS), (size_t)C::SMEM, dev.stream, tq, tk, tv, p, static_cast<bf16*>(out),
                    1.4426950408889634f / sqrtf((float)HD), sync, static_cast<float*>(scratch), dev.err, kWaitTimeoutNs);
}

}  // namespace

bool paged_tc_takes(const Paged& p) { return p.Hq / p.Hkv <= kPtRows; }

size_t paged_tc_scratch(const Paged& p) {
  return (size_t)kPtMaxCtas * 2 * (p.hd == 128 ? PtCfg<128, false>::PART : PtCfg<64, false>::PART) * 4;
}

cudaError_t paged_tc(const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch, const Dev& dev) {
  if (p.hd == 128)
    return p.i8 ? launch_tc<128, true>(p, q, ld_q, out, sync, scratch, dev)
                : launch_tc<128, false>(p, q, ld_q, out, sync, scratch, dev);
  return p.i8 ? launch_tc<64, true>(p, q, ld_q, out, sync, scratch, dev)
              : launch_tc<64, false>(p, q, ld_q, out, sync, scratch, dev);
}

}  // namespace adadsf
