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

// A line of tiles of keys, shared out in equal pieces. Sequence b's items run group of rows by
// group of rows, key/value heads inside. An item takes PAD places (what its start and
// end cost) and then one for each tile of the keys that its last row sees (at least one). The places
// of a piece are its CTA's work; items of at most WHOLE tiles are not cut, they go to the
// CTA that has their first tile. CUT: rows of a group (groups, tokens), keys of a tile (KEYS), PAD, WHOLE.
// A warp keeps 32 sequences at a time, one a lane.
template <class CUT>
struct PagedItem {
  int b, h, grp, n, len, tiles, seen;  // seen: keys that its last row sees
  int64_t row0, at0;                   // first packed row of the sequence, place of the first tile
  // its tiles [j0, j1) in the piece [ua, ub)
  __device__ __forceinline__ void in(int64_t ua, int64_t ub, int* j0, int* j1) const {
    if (tiles <= CUT::WHOLE) {
      *j0 = 0;
      *j1 = at0 >= ua && at0 < ub ? tiles : 0;
    } else {
      *j0 = (int)max((int64_t)0, ua - at0);
      *j1 = (int)min((int64_t)tiles, ub - at0);
    }
  }
  // the CTAs that have its first tile and tile number `last` (the same where it is not cut)
  __device__ __forceinline__ int first_cta(int64_t per) const { return (int)(at0 / per); }
  __device__ __forceinline__ int last_cta(int64_t per, int last) const {
    return (int)((tiles <= CUT::WHOLE ? at0 : at0 + last) / per);
  }
};
template <class CUT>
struct PagedLine {
  CUT cut;
  int64_t base, end;      // of this chunk of sequences on the line
  int b0;
  PagedSeq q;             // this lane's sequence
  int64_t mine, at;       // its tiles, and their place on the line
  int b, grp;             // the group that item() found last, and its place
  int64_t x;

  static __device__ __forceinline__ int tiles_of(int seen) { return seen <= CUT::KEYS ? 1 : (seen + CUT::KEYS - 1) / CUT::KEYS; }
  // keys that the last row of group g sees
  __device__ __forceinline__ int seen_of(int n, int len, int g) const { return max(0, len - n + min(n, cut.tokens(g))); }
  __device__ __forceinline__ void load(const Paged& p, int b_first, int64_t from, int lane, int* err) {
    b0 = b_first;
    b = -1;
    base = from;
    q = PagedSeq{0, 0, 0};
    mine = 0;
    if (b0 + lane < p.B) {
      q = paged_seq(p, b0 + lane, err);
      const int groups = cut.groups(q.n);
      for (int g = 0; g < groups; ++g) mine += CUT::PAD + tiles_of(seen_of(q.n, q.len, g));
      mine *= p.Hkv;
    }
    int64_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    at = base + inc - mine;
    end = base + __shfl_sync(0xffffffffu, inc, 31);
  }
  // [first, last) of CTA `cta` of `ctas` in pieces of *per places, `least` or more
  __device__ __forceinline__ void piece(const Paged& p, int least, int cta, int ctas, int lane, int* err, int64_t* per,
                                        int64_t* first, int64_t* last) {
    int64_t all = 0;
    for (int c = 0; c < p.B; c += 32) {
      load(p, c, all, lane, err);
      all = end;
    }
    *per = max((int64_t)least, (all + ctas - 1) / ctas);
    *first = min(all, cta * *per);
    *last = min(all, *first + *per);
    if (*first < base) load(p, 0, 0, lane, err);
  }
  // the item that holds place *u (below the line's length; calls with rising *u), which moves past it
  __device__ __forceinline__ PagedItem<CUT> item(const Paged& p, int64_t* to, int lane, int* err) {
    const int64_t u = *to;
    while (u >= end) load(p, b0 + 32, end, lane, err);
    const int l = __ffs(__ballot_sync(0xffffffffu, u >= at && u < at + mine)) - 1;
    PagedItem<CUT> it;
    it.b = b0 + l;
    it.n = __shfl_sync(0xffffffffu, q.n, l);
    it.len = __shfl_sync(0xffffffffu, q.len, l);
    it.row0 = __shfl_sync(0xffffffffu, q.row0, l);
    const int64_t from = __shfl_sync(0xffffffffu, at, l);
    if (b != it.b) {
      b = it.b;
      grp = 0;
      x = from;
    }
    for (;; ++grp) {
      it.seen = seen_of(it.n, it.len, grp);
      it.tiles = tiles_of(it.seen);
      const int64_t all = (int64_t)(CUT::PAD + it.tiles) * p.Hkv;
      if (u < x + all) break;
      x += all;
    }
    it.grp = grp;
    it.h = (int)((u - x) / (CUT::PAD + it.tiles));
    it.at0 = x + (int64_t)it.h * (CUT::PAD + it.tiles) + CUT::PAD;
    *to = it.at0 + it.tiles;
    return it;
  }
};

// Waits that poll: a suspended thread is woken late (all of the kernel's waits with a suspension
// of up to 100 us took 430 us where these take 404, at 2048 tokens on 14336 of 28 heads).
__device__ __forceinline__ bool paged_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool paged_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* err, unsigned long long timeout_ns) {
  if (paged_try(bar, parity)) return true;
  const unsigned long long t0 = globaltimer_ns();
  for (uint32_t it = 1;; ++it) {
    if (paged_try(bar, parity)) return true;
    if ((it & 63u) == 0) {
      if (*abort_flag) return false;
      if (globaltimer_ns() - t0 > timeout_ns) {
        *abort_flag = 1;
        set_device_error(err, DEVERR_TIMEOUT);
        return false;
      }
    }
  }
}

// Two 8-bit numbers (the low bytes of t's halves) as bf16, exactly: with b a number's low seven
// bits and s its top one, (128 + b) - (s ? 256 : 128).
__device__ __forceinline__ uint32_t bf16_of_i8(uint32_t t) {
  const uint32_t b = (t & 0x007f007fu) | 0x43004300u, s = (t & 0x00800080u) | 0x43004300u;
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&b), *reinterpret_cast<const __nv_bfloat162*>(&s));
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}

}  // namespace adadsf
