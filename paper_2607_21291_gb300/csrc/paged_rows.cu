// Attention of few new tokens over a paged cache, bf16 (adadsf_paged_attention): 16
// packed rows (token i's G query heads of a key/value head side by side, row i G + g) against
// tiles of 64 keys.
//
// What bounds it is reading the cache, once per 16 rows. One CTA is four consumer warps and
// a producer warp that streams tiles through a ring by TMA, a box a page (128- or
// 64-byte swizzle), 8-bit tiles with their scales by bulk copies. A consumer warp takes 16
// keys of a tile:
//   S (16 x 16) = Q (16 x hd) K^T         m16n8k16 products; the order of the features in a
//                                         k step is free, so a lane's operands come from whole
//                                         16-byte chunks of a key
//   online softmax per row                fp32, base 2
//   O (16 x hd) += P (16 x 16) V          P as bf16 and a bf16 of what that leaves: reading is
//                                         what takes the time, and rounded weights would add
//                                         an error as large as the output's rounding
// 8-bit numbers become bf16 exactly in registers (bf16_of_i8: a byte permutation, two logic
// operations and a subtraction for two). Key scales multiply scores, value scales weights.
//
// All tiles of all (sequence, row tile, key/value head) items lie on one line that is cut
// into equal pieces, one per CTA: any mix of lengths fills the machine. An item cut in
// pieces leaves fp32 partials in the workspace; the CTA that finishes last joins them in the
// order of the pieces (a counter in the synchronisation area, left at zero), so the
// result does not depend on which one that is. Its four warps take a quarter of the features
// each: one single token on 131071 cached has 77 pieces a head to join (95 us with one warp).
//
// Measured, 28 query heads on 4 of 128: 8 single tokens on 32767 cached 89 us, 6.0 TB/s (89% of
// a plain copy); 8-bit numbers 94 us, 2.9 TB/s, bound by the instructions that make them
// bf16; 16 on up to 4096 in 8 bits 22 us; one on 131071 70 us (8 bits 73); 256 on 300 44 us (49).
#include <math.h>

#include <algorithm>

#include "paged.cuh"

namespace adadsf {
namespace {

constexpr int kPrRows = 16;               // packed rows of an item
constexpr int kPrWarps = 4;               // consumer warps, a quarter of a tile's keys each
constexpr int kPrThreads = 32 * (kPrWarps + 1);
constexpr int kPrPerSm = 2;               // CTAs an SM (three, of 128 registers a thread: 8 to 10% slower)
constexpr int kPrMaxCtas = 160 * kPrPerSm;
constexpr int kPrPad = 2;                 // an item's start and end, in tiles
constexpr int kPrWhole = 8;               // tiles up to which an item is not cut
constexpr int kPrMin = 4;                 // fewest places of a piece

template <int HD, bool I8>
struct PrCfg {
  static constexpr int KPW = 16;                           // keys of a warp's step, a quarter of a tile (32: longer code, no faster)
  static constexpr int TK = kPrWarps * KPW;                // keys of a tile
  static constexpr int STAGES = I8 || HD == 64 ? 5 : 3;
  static constexpr int SLABS = I8 ? 1 : HD / 64;           // 128-byte (8-bit, hd 64: 64-byte) wide parts of a row
  static constexpr int ROWB = I8 ? HD : 128;               // bytes of a row in a slab
  static constexpr int TILE = SLABS * TK * ROWB;           // K or V of a stage
  static constexpr int SCALES = I8 ? 2 * TK * 4 : 0;       // K scales, V scales
  static constexpr int STAGE = 2 * TILE + (I8 ? 1024 : 0);  // tiles stay 1024-byte aligned
  static constexpr int QF = HD / 32 * 2 * 32 * 16;         // the item's queries as A operands
  static constexpr int SMEM = STAGES * STAGE + QF + 1024;
  static constexpr int MERGE = HD / 8 * 32 * 16;           // one warp's O
  static_assert(SCALES <= 1024 && 2 * MERGE <= 2 * TILE, "two warps' O fit the stage they free");
};

__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float2 lds_f2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
  return v;
}
// Groups of 16 packed rows, tiles of TK keys.
template <int TK>
struct PrCut {
  static constexpr int KEYS = TK, PAD = kPrPad, WHOLE = kPrWhole;
  int G;
  __device__ __forceinline__ int groups(int n) const { return (int)(((int64_t)n * G + kPrRows - 1) / kPrRows); }
  __device__ __forceinline__ int tokens(int g) const { return (int)((((int64_t)g + 1) * kPrRows - 1) / G) + 1; }
};

template <int HD, bool I8>
__global__ void __launch_bounds__(kPrThreads, kPrPerSm)
    paged_rows_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv, const Paged p,
                      const bf16* q, int64_t ld_q, bf16* out, float scale_log2, int* sync, float* parts, int* err,
                      unsigned long long timeout_ns) {
  using C = PrCfg<HD, I8>;
  using Cut = PrCut<C::TK>;
  constexpr int KPW = C::KPW, TK = C::TK, KT = KPW / 8;   // a warp's keys of a tile, in n tiles
  constexpr int NT = HD / 8;                    // n tiles of the output
  constexpr int SLOT = kPrRows * HD + 64;       // floats of a partial: O (per lane and n tile), then (m, l)
  extern __shared__ __align__(1024) uint8_t dsm[];
  __shared__ __align__(8) uint64_t bars[2 * C::STAGES];
  __shared__ float2 ml_s[2][kPrRows];           // (m, l) of the merging warps
  __shared__ int abort_s, failed_s, done_s;
  const uint32_t ring = (smem_u32(dsm) + 1023u) & ~1023u;
  uint8_t* ring_p = dsm + (ring - smem_u32(dsm));
  const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[C::STAGES]);
  volatile int* abort_flag = &abort_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = p.Hq / p.Hkv;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(full0 + 8 * i, 1);
      mbar_init(empty0 + 8 * i, kPrWarps);
    }
    abort_s = failed_s = 0;
    fence_barrier_init();
  }
  if (warp == kPrWarps && lane == 0) {
    tma_prefetch_desc(&tk);
    tma_prefetch_desc(&tv);
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  // this CTA's piece of the line
  PagedLine<Cut> line{Cut{G}};
  int64_t per, ua, ub;
  line.piece(p, kPrMin, (int)blockIdx.x, (int)gridDim.x, lane, err, &per, &ua, &ub);
  if (ua >= ub) return;

  if (warp == kPrWarps) {
    // ------------------------------------------------------------ producer
    const int box = min(1 << p.page_log2, TK), boxes = TK / box;   // rows of a copy, copies of a tile
    int issued = 0;
    bool ok = true;
    for (int64_t u = ua; ok && u < ub;) {
      const PagedItem<Cut> it = line.item(p, &u, lane, err);
      int t, t1;
      it.in(ua, ub, &t, &t1);
      if (it.seen == 0 || t >= t1) continue;
      const int32_t* tab = p.table + (int64_t)it.b * p.max_pages;
      // a lane's page of tile t; pages past the last visible key are not looked at
      auto page_of = [&](int t) {
        const int place = t * TK + lane * box;
        return lane < boxes && place < it.seen ? tab[place >> p.page_log2] : 0;
      };
      int next = page_of(t);
      for (; t < t1; ++t) {
        const int st = issued % C::STAGES;
        const int page = next;
        if (t + 1 < t1) next = page_of(t + 1);
        const int place = t * TK + lane * box;
        const bool want = lane < boxes && place < it.seen;
        const bool there = (unsigned)page < (unsigned)p.n_pages;
        if (want && !there) set_device_error(err, DEVERR_INDEX);
        int w = 0;
        if (lane == 0) w = paged_wait(empty0 + 8 * st, ((issued / C::STAGES) & 1) ^ 1, abort_flag, err, timeout_ns);
        if (!__shfl_sync(0xffffffffu, w, 0)) { ok = false; break; }
        const uint32_t dk = ring + st * C::STAGE, ds = dk + 2 * C::TILE, fb = full0 + 8 * st;
        const unsigned wants = __ballot_sync(0xffffffffu, want), good = __ballot_sync(0xffffffffu, want && there);
        if (I8 && want && !there) {   // a page that is not: zeros, scales too
          float* sc = reinterpret_cast<float*>(ring_p + st * C::STAGE + 2 * C::TILE);
          for (int i = 0; i < box; ++i) sc[lane * box + i] = sc[TK + lane * box + i] = 0.f;
        }
        __syncwarp();
        if (lane == 0)
          mbar_arrive_expect_tx(fb, (uint32_t)(__popc(wants) * box * C::SLABS * C::ROWB * 2 +
                                               (I8 ? __popc(good) * box * 8 : 0)));
        __syncwarp();
        if (want) {
          // out of the pool: the copy fills with zeros
          const int z = there ? page * p.Hkv + it.h : p.n_pages * p.Hkv;
          const int r = place & ((1 << p.page_log2) - 1);
#pragma unroll
          for (int x = 0; x < C::SLABS; ++x) {
            const uint32_t o = x * TK * C::ROWB + lane * box * C::ROWB;
            tma_load_3d(dk + o, &tk, x * 64, r, z, fb);
            tma_load_3d(dk + C::TILE + o, &tv, x * 64, r, z, fb);
          }
          if (I8 && there) {
            const int64_t vec = ((int64_t)z << p.page_log2) + r;
            bulk_load(ds + lane * box * 4, p.ks + vec, box * 4, fb);
            bulk_load(ds + TK * 4 + lane * box * 4, p.vs + vec, box * 4, fb);
          }
        }
        ++issued;
      }
    }
    // drain: the copies issued last into each stage have landed
    if (lane == 0)
      for (int st = 0; st < C::STAGES && st < issued; ++st) {
        const int last = st + ((issued - 1 - st) / C::STAGES) * C::STAGES;
        mbar_wait_drain(full0 + 8 * st, (uint32_t)((last / C::STAGES) & 1), timeout_ns);
      }
    return;
  }
  // -------------------------------------------------------------- consumers
  const int gid = lane >> 2, tig = lane & 3;
  const int mi = lane >> 3, mr = lane & 7;   // ldmatrix: this lane's matrix and row
  int taken = 0;
  for (int64_t u = ua; u < ub;) {
    const PagedItem<Cut> it = line.item(p, &u, lane, err);
    int t0, t1;
    it.in(ua, ub, &t0, &t1);
    if (t0 >= t1) continue;
    // rows gid and gid + 8: their token and head, and the keys that they see
    const bf16* src[2];
    bf16* dst[2];
    int lim[2];
    bool live[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int x = it.grp * kPrRows + gid + 8 * r, i = x / G, g = x - i * G;
      live[r] = i < it.n;
      lim[r] = live[r] ? it.len - it.n + i + 1 : 0;
      src[r] = q + (it.row0 + i) * ld_q + (it.h * G + g) * HD;
      dst[r] = out + ((it.row0 + i) * p.Hq + it.h * G + g) * HD;
    }
    if (it.seen == 0) {   // nothing to attend to (one tile on the line, so one piece)
#pragma unroll
      for (int r = 0; r < 2; ++r)
        if (live[r] && warp == 0)
          for (int e = tig * (HD / 4); e < (tig + 1) * (HD / 4); e += 8)
            *reinterpret_cast<uint4*>(dst[r] + e) = make_uint4(0, 0, 0, 0);
      continue;
    }
    // Q as A operands in shared memory (registers for them would cost a CTA an SM): part n of a lane is a 16-byte
    // chunk of row gid or gid + 8 whose words pair with those of the keys' chunks (bf16: chunk 2 tig + i of slab s;
    // 8 bits: halves of 16 features)
    constexpr int QN = HD / 32;
    uint4* sq = reinterpret_cast<uint4*>(ring_p + C::STAGES * C::STAGE);
#pragma unroll
    for (int n = 0; n < QN; ++n) {
      if (n % kPrWarps != warp) continue;
      const int at = I8 ? 16 * (HD / 64 * tig + n / 2) + 8 * (n & 1) : 64 * (n / 2) + 8 * (2 * tig + (n & 1));
#pragma unroll
      for (int r = 0; r < 2; ++r)
        sq[(2 * n + r) * 32 + lane] = live[r] ? *reinterpret_cast<const uint4*>(src[r] + at) : make_uint4(0, 0, 0, 0);
    }
    named_bar_sync(1, 32 * kPrWarps);
    float o[NT][4];
    float m_r[2] = {-INFINITY, -INFINITY}, l_r[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    // keys that every row of the item sees: tiles below need no mask
    const int open = it.len - it.n + it.grp * kPrRows / G + 1;
    bool ok = true;
    int st = 0;
    for (int t = t0; t < t1; ++t, ++taken) {
      st = taken % C::STAGES;
      ok = paged_wait(full0 + 8 * st, (taken / C::STAGES) & 1, abort_flag, err, timeout_ns);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const uint32_t kt = ring + st * C::STAGE, vt = kt + C::TILE, ks = kt + 2 * C::TILE, vs = ks + TK * 4;
      const int kw = warp * KPW;                            // this warp's keys within the tile
      const int j0 = t * TK + kw;
      if (j0 < it.seen) {
        float sc[KT][4];
#pragma unroll
        for (int nt = 0; nt < KT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
        // a loop: the tile's code is long for the instruction caches
#pragma unroll 2
        for (int n = 0; n < QN; n += 2) {
          const uint4 a0 = sq[(2 * n) * 32 + lane], a1 = sq[(2 * n + 1) * 32 + lane];
          const uint4 a2 = sq[(2 * n + 2) * 32 + lane], a3 = sq[(2 * n + 3) * 32 + lane];
#pragma unroll
          for (int nt = 0; nt < KT; ++nt) {
            const int row = kw + 8 * nt + gid;
            if (I8) {
              const int c = HD / 64 * tig + n / 2;
              const uint4 k4 = HD == 128 ? lds128(kt + row * 128 + ((c ^ (row & 7)) << 4))
                                         : lds128(kt + row * 64 + ((c ^ ((row >> 1) & 3)) << 4));
              auto half = [&](uint32_t w, uint32_t sel) { return bf16_of_i8(__byte_perm(w, 0, sel)); };
              mma_16816(sc[nt], a0.x, a1.x, a0.y, a1.y, half(k4.x, 0x4140), half(k4.x, 0x4342));
              mma_16816(sc[nt], a0.z, a1.z, a0.w, a1.w, half(k4.y, 0x4140), half(k4.y, 0x4342));
              mma_16816(sc[nt], a2.x, a3.x, a2.y, a3.y, half(k4.z, 0x4140), half(k4.z, 0x4342));
              mma_16816(sc[nt], a2.z, a3.z, a2.w, a3.w, half(k4.w, 0x4140), half(k4.w, 0x4342));
            } else {
              const uint32_t at = kt + (n / 2) * TK * 128 + row * 128;
              const uint4 k4 = lds128(at + (((2 * tig) ^ (row & 7)) << 4)), k5 = lds128(at + (((2 * tig + 1) ^ (row & 7)) << 4));
              mma_16816(sc[nt], a0.x, a1.x, a0.y, a1.y, k4.x, k4.y);
              mma_16816(sc[nt], a0.z, a1.z, a0.w, a1.w, k4.z, k4.w);
              mma_16816(sc[nt], a2.x, a3.x, a2.y, a3.y, k5.x, k5.y);
              mma_16816(sc[nt], a2.z, a3.z, a2.w, a3.w, k5.z, k5.w);
            }
          }
        }
        // online softmax over the warp's keys; score [nt][2 r + e] is row gid + 8 r, key j0 + 8 nt + 2 tig + e
        float2 vsc[KT];
#pragma unroll
        for (int nt = 0; nt < KT; ++nt) {
          float2 k2 = make_float2(scale_log2, scale_log2);
          if (I8) {
            const float2 kk = lds_f2(ks + 4 * (kw + 8 * nt + 2 * tig));
            vsc[nt] = lds_f2(vs + 4 * (kw + 8 * nt + 2 * tig));
            k2.x *= kk.x;
            k2.y *= kk.y;
          }
          sc[nt][0] *= k2.x; sc[nt][1] *= k2.y; sc[nt][2] *= k2.x; sc[nt][3] *= k2.y;
        }
        const bool masked = j0 + KPW > open;
        if (masked) {
#pragma unroll
          for (int nt = 0; nt < KT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (j0 + 8 * nt + 2 * tig + (e & 1) >= lim[e >> 1]) sc[nt][e] = -INFINITY;
        }
        float corr[2], base[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float mx = fmaxf(sc[0][2 * r], sc[0][2 * r + 1]);
#pragma unroll
          for (int nt = 1; nt < KT; ++nt) mx = fmaxf(mx, fmaxf(sc[nt][2 * r], sc[nt][2 * r + 1]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          const float mn = fmaxf(m_r[r], mx);
          base[r] = mn == -INFINITY ? 0.f : mn;
          corr[r] = ex2_approx(m_r[r] - base[r]);
          m_r[r] = mn;
        }
        uint32_t pa[2 * KT], pl[2 * KT];   // weights: bf16, and what that leaves
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float sum = 0.f;
#pragma unroll
          for (int nt = 0; nt < KT; ++nt) {
            float p0 = ex2_approx(sc[nt][2 * r] - base[r]), p1 = ex2_approx(sc[nt][2 * r + 1] - base[r]);
            sum += p0 + p1;
            if (I8) {
              p0 *= vsc[nt].x;
              p1 *= vsc[nt].y;
            }
            const uint32_t two = pack_bf16x2(p0, p1);
            pa[2 * nt + r] = two;
            pl[2 * nt + r] = pack_bf16x2(p0 - __uint_as_float(two << 16), p1 - __uint_as_float(two & 0xffff0000u));
          }
          l_r[r] = l_r[r] * corr[r] + sum;
        }
        if (I8 && masked) {   // the scale of a key that a row does not see may be anything, and zero times it is not always zero
#pragma unroll
          for (int nt = 0; nt < KT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int key = j0 + 8 * nt + 2 * tig;
              const uint32_t sees = (key < lim[r] ? 0xffffu : 0u) | (key + 1 < lim[r] ? 0xffff0000u : 0u);
              pa[2 * nt + r] &= sees;
              pl[2 * nt + r] &= sees;
            }
        }
        if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            o[j][0] *= corr[0]; o[j][1] *= corr[0];
            o[j][2] *= corr[1]; o[j][3] *= corr[1];
          }
        }
        if (I8) {
          // keys 2 tig, 2 tig + 1, 2 tig + 8, 2 tig + 9; n tile j holds feature NT gid + j in column gid
          if (HD == 128) {
            uint4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int row = kw + 2 * tig + (k & 1) + 8 * (k >> 1);
              v[k] = lds128(vt + row * 128 + ((gid ^ (row & 7)) << 4));
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              auto word = [&](int k) { return w == 0 ? v[k].x : w == 1 ? v[k].y : w == 2 ? v[k].z : v[k].w; };
#pragma unroll
              for (int f = 0; f < 4; ++f) {
                const uint32_t sel = 0x4400u + f * 0x1111u;   // byte f of either key
                const uint32_t b0 = bf16_of_i8(__byte_perm(word(0), word(1), sel)), b1 = bf16_of_i8(__byte_perm(word(2), word(3), sel));
                mma_16816(o[4 * w + f], pa[0], pa[1], pa[2], pa[3], b0, b1);
                mma_16816(o[4 * w + f], pl[0], pl[1], pl[2], pl[3], b0, b1);
              }
            }
          } else {
            uint2 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int row = kw + 2 * tig + (k & 1) + 8 * (k >> 1);
              v[k] = lds64(vt + row * 64 + (((gid >> 1) ^ ((row >> 1) & 3)) << 4) + ((gid & 1) << 3));
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              auto word = [&](int k) { return w == 0 ? v[k].x : v[k].y; };
#pragma unroll
              for (int f = 0; f < 4; ++f) {
                const uint32_t sel = 0x4400u + f * 0x1111u;   // byte f of either key
                const uint32_t b0 = bf16_of_i8(__byte_perm(word(0), word(1), sel)), b1 = bf16_of_i8(__byte_perm(word(2), word(3), sel));
                mma_16816(o[4 * w + f], pa[0], pa[1], pa[2], pa[3], b0, b1);
                mma_16816(o[4 * w + f], pl[0], pl[1], pl[2], pl[3], b0, b1);
              }
            }
          }
        } else {
          // V of a key that a row does not see may be anything, and zero times it is not always
          // zero: keys from `open` on stay out of the products and go to their rows below
          uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
          if (masked) {
            const int k0 = j0 + 2 * tig;
            keep0 = (k0 < open ? 0xffffu : 0u) | (k0 + 1 < open ? 0xffff0000u : 0u);
            keep1 = (k0 + 8 < open ? 0xffffu : 0u) | (k0 + 9 < open ? 0xffff0000u : 0u);
          }
#pragma unroll
          for (int np = 0; np < HD / 16; ++np) {
            uint32_t vb[4];
            const int row = kw + (mi & 1) * 8 + mr, col = np * 16 + (mi >> 1) * 8;
            ldmatrix_x4_trans(vt + (col >> 6) * TK * 128 + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4), vb);
            if (masked) { vb[0] &= keep0; vb[1] &= keep1; vb[2] &= keep0; vb[3] &= keep1; }
            mma_16816(o[2 * np], pa[0], pa[1], pa[2], pa[3], vb[0], vb[1]);
            mma_16816(o[2 * np + 1], pa[0], pa[1], pa[2], pa[3], vb[2], vb[3]);
            mma_16816(o[2 * np], pl[0], pl[1], pl[2], pl[3], vb[0], vb[1]);
            mma_16816(o[2 * np + 1], pl[0], pl[1], pl[2], pl[3], vb[2], vb[3]);
          }
          for (int key = max(open, j0); key < min(it.seen, j0 + KPW); ++key) {
            const int x = key - j0, row = kw + x;
            float w[2];   // the weight as the products take it
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int from = (lane & 28) | ((x & 7) >> 1);
              uint32_t hi = x < 8 ? pa[r] : pa[2 + r], lo = x < 8 ? pl[r] : pl[2 + r];
              hi = __shfl_sync(0xffffffffu, hi, from);
              lo = __shfl_sync(0xffffffffu, lo, from);
              w[r] = (x & 1) ? __uint_as_float(hi & 0xffff0000u) + __uint_as_float(lo & 0xffff0000u)
                             : __uint_as_float(hi << 16) + __uint_as_float(lo << 16);
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              const uint32_t two = *reinterpret_cast<const uint32_t*>(
                  ring_p + (vt - ring) + (j >> 3) * TK * 128 + row * 128 + (((j & 7) ^ (row & 7)) << 4) + 4 * tig);
              const float v0 = __uint_as_float(two << 16), v1 = __uint_as_float(two & 0xffff0000u);
              if (key < lim[0]) { o[j][0] = fmaf(w[0], v0, o[j][0]); o[j][1] = fmaf(w[0], v1, o[j][1]); }
              if (key < lim[1]) { o[j][2] = fmaf(w[1], v0, o[j][2]); o[j][3] = fmaf(w[1], v1, o[j][3]); }
            }
          }
        }
      }
      if (t + 1 < t1) {   // the piece's last stage is kept for the merge
        __syncwarp();
        if (lane == 0) mbar_arrive(empty0 + 8 * st);
      }
    }
    if (!ok && lane == 0) *(volatile int*)&failed_s = 1;   // the warps leave together, after the barrier
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l_r[r] += __shfl_xor_sync(0xffffffffu, l_r[r], 1);
      l_r[r] += __shfl_xor_sync(0xffffffffu, l_r[r], 2);
    }
    // the four warps' results into warp 0's: 2 and 3 hand theirs to 0 and 1, then 1 to 0
    float4* area = reinterpret_cast<float4*>(ring_p + st * C::STAGE);
    auto give = [&](int slot) {
#pragma unroll
      for (int j = 0; j < NT; ++j) area[(slot * NT + j) * 32 + lane] = make_float4(o[j][0], o[j][1], o[j][2], o[j][3]);
      if (tig == 0) {
        ml_s[slot][gid] = make_float2(m_r[0], l_r[0]);
        ml_s[slot][gid + 8] = make_float2(m_r[1], l_r[1]);
      }
    };
    // (m, l, O) joined with another's: weights 2^(m - max) of either side
    auto join_ml = [&](const float2 (&ml)[2], float (&mine)[2], float (&theirs)[2]) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float mn = fmaxf(m_r[r], ml[r].x), b = mn == -INFINITY ? 0.f : mn;
        mine[r] = ex2_approx(m_r[r] - b);
        theirs[r] = ex2_approx(ml[r].x - b);
        l_r[r] = l_r[r] * mine[r] + ml[r].y * theirs[r];
        m_r[r] = mn;
      }
    };
    auto join_o = [&](int j, const float4& x, const float (&mine)[2], const float (&theirs)[2]) {
      o[j][0] = o[j][0] * mine[0] + x.x * theirs[0];
      o[j][1] = o[j][1] * mine[0] + x.y * theirs[0];
      o[j][2] = o[j][2] * mine[1] + x.z * theirs[1];
      o[j][3] = o[j][3] * mine[1] + x.w * theirs[1];
    };
    auto take = [&](int slot) {
      const float2 ml[2] = {ml_s[slot][gid], ml_s[slot][gid + 8]};
      float mine[2], theirs[2];
      join_ml(ml, mine, theirs);
#pragma unroll
      for (int j = 0; j < NT; ++j) join_o(j, area[(slot * NT + j) * 32 + lane], mine, theirs);
    };
    named_bar_sync(1, 32 * kPrWarps);   // the stage is read by all
    if (*(volatile int*)&failed_s) return;
    if (warp >= 2) give(warp - 2);
    named_bar_sync(1, 32 * kPrWarps);
    if (warp < 2) take(warp);
    named_bar_sync(1, 32 * kPrWarps);
    if (warp == 1) give(0);
    named_bar_sync(1, 32 * kPrWarps);
    if (warp == 0) take(0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // written by threads, next by a copy
    __syncwarp();
    if (lane == 0) mbar_arrive(empty0 + 8 * st);
    // warp 0 holds the piece's result
    // a row's 1 / l; a row without a key is zero, and one whose keys are all -inf or one of them NaN is NaN
    auto inv_of = [&](int r) { return l_r[r] > 0.f ? 1.f / l_r[r] : lim[r] > 0 ? l_r[r] / l_r[r] : 0.f; };
    if (t0 == 0 && t1 == it.tiles) {
      if (warp != 0) continue;
      if (I8) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (!live[r]) continue;
          const float inv = inv_of(r);
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < NT; j += 8) {
              float f[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) f[k] = o[j + k][2 * r + e] * inv;
              store_vec(dst[r] + NT * (2 * tig + e) + j, f);
            }
        }
      } else {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (!live[r]) continue;
          const float inv = inv_of(r);
#pragma unroll
          for (int j = 0; j < NT; ++j)
            *reinterpret_cast<uint32_t*>(dst[r] + 8 * j + 2 * tig) = pack_bf16x2(o[j][2 * r] * inv, o[j][2 * r + 1] * inv);
        }
      }
      continue;
    }
    const int first = it.first_cta(per), last = it.last_cta(per, it.tiles - 1);
    auto slot_of = [&](int cta) { return parts + ((int64_t)cta * 2 + (cta == first ? 1 : 0)) * SLOT; };
    if (warp == 0) {
      float* mine = slot_of((int)blockIdx.x);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        __stcg(reinterpret_cast<float4*>(mine) + j * 32 + lane, make_float4(o[j][0], o[j][1], o[j][2], o[j][3]));
      if (tig == 0) {
        __stcg(reinterpret_cast<float2*>(mine + kPrRows * HD) + gid, make_float2(m_r[0], l_r[0]));
        __stcg(reinterpret_cast<float2*>(mine + kPrRows * HD) + gid + 8, make_float2(m_r[1], l_r[1]));
      }
      __threadfence();
      __syncwarp();
      if (lane == 0) {
        const int done = atomicAdd(sync + first, 1) == last - first;
        if (done) sync[first] = 0;
        *(volatile int*)&done_s = done;
        __threadfence();
      }
    }
    named_bar_sync(1, 32 * kPrWarps);
    const bool done = *(volatile int*)&done_s != 0;
    named_bar_sync(1, 32 * kPrWarps);   // read before the next item's
    if (!done) continue;
    // the last one to finish joins the pieces, a quarter of the n tiles a warp, four pieces at a time
    __threadfence();
    constexpr int NW = NT / kPrWarps;
    float4 sum[NW];
#pragma unroll
    for (int j = 0; j < NW; ++j) sum[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    m_r[0] = m_r[1] = -INFINITY;
    l_r[0] = l_r[1] = 0.f;
    for (int c = first; c <= last; c += 4) {
      float4 x[4][NW];
      float2 ml[4][2];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* from = slot_of(min(c + k, last));
#pragma unroll
        for (int j = 0; j < NW; ++j) x[k][j] = __ldcg(reinterpret_cast<const float4*>(from) + (warp * NW + j) * 32 + lane);
#pragma unroll
        for (int r = 0; r < 2; ++r) ml[k][r] = __ldcg(reinterpret_cast<const float2*>(from + kPrRows * HD) + gid + 8 * r);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (c + k > last) break;
        float mine[2], theirs[2];
        join_ml(ml[k], mine, theirs);
#pragma unroll
        for (int j = 0; j < NW; ++j)
          sum[j] = make_float4(sum[j].x * mine[0] + x[k][j].x * theirs[0], sum[j].y * mine[0] + x[k][j].y * theirs[0],
                               sum[j].z * mine[1] + x[k][j].z * theirs[1], sum[j].w * mine[1] + x[k][j].w * theirs[1]);
      }
    }
    // n tile j: features 8 j + 2 tig + e, or (8 bits) NT (2 tig + e) + j
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      if (!live[r]) continue;
      const float inv = inv_of(r);
#pragma unroll
      for (int j = 0; j < NW; ++j) {
        const float a = (r ? sum[j].z : sum[j].x) * inv, b = (r ? sum[j].w : sum[j].y) * inv;
        bf16* to = dst[r] + (I8 ? NT * 2 * tig + warp * NW + j : 8 * (warp * NW + j) + 2 * tig);
        if (I8) {
          to[0] = __float2bfloat16_rn(a);
          to[NT] = __float2bfloat16_rn(b);
        } else {
          *reinterpret_cast<uint32_t*>(to) = pack_bf16x2(a, b);
        }
      }
    }
  }
}

template <int HD, bool I8>
cudaError_t launch_rows(const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch, const Dev& dev) {
  using C = PrCfg<HD, I8>;
  const cudaError_t e = allow_smem<paged_rows_kernel<HD, I8>, C::SMEM>();
  if (e != cudaSuccess) return e;
  CUtensorMap tk, tv;
  if (!make_tmap_pages(&tk, p.k, p, I8, C::TK) || !make_tmap_pages(&tv, p.v, p, I8, C::TK)) return cudaErrorInvalidValue;
  // no more CTAs than pieces of the fewest tiles that any counts could make
  const int G = p.Hq / p.Hkv;
  const int64_t span = ((int64_t)p.max_pages << p.page_log2) / C::TK + 1;
  const int64_t row_tiles = std::min<int64_t>((int64_t)p.B * ((p.max_new * (int64_t)G + kPrRows - 1) / kPrRows),
                                              p.n_rows * G);
  const int64_t most = std::max<int64_t>(1, (row_tiles * p.Hkv * (span + kPrPad) + kPrMin - 1) / kPrMin);
  const int64_t room = std::min(dev.num_sms * kPrPerSm, kPrMaxCtas);
  return launch_pdl(paged_rows_kernel<HD, I8>, dim3((unsigned)std::min(most, room)), dim3(kPrThreads), (size_t)C::SMEM,
                    dev.stream, tk, tv, p, static_cast<const bf16*>(q), ld_q, static_cast<bf16*>(out),
                    1.4426950408889634f / sqrtf((float)HD), sync, static_cast<float*>(scratch), dev.err, kWaitTimeoutNs);
}

}  // namespace

size_t paged_rows_scratch(const Paged& p) { return (size_t)kPrMaxCtas * 2 * (kPrRows * p.hd + 64) * 4; }

cudaError_t paged_rows(const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch, const Dev& dev) {
  if (p.hd == 128)
    return p.i8 ? launch_rows<128, true>(p, q, ld_q, out, sync, scratch, dev)
                : launch_rows<128, false>(p, q, ld_q, out, sync, scratch, dev);
  return p.i8 ? launch_rows<64, true>(p, q, ld_q, out, sync, scratch, dev)
              : launch_rows<64, false>(p, q, ld_q, out, sync, scratch, dev);
}

}  // namespace adadsf
