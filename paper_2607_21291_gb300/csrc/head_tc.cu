// Products of the losses at the LM head on the 5th-generation tensor cores.
//
// One persistent kernel, a CTA pair a tile of 256 x 256 (tcgen05.mma cta_group::2, fp32
// accumulators in TMEM, two of them, so that one tile's epilogue runs under the next one's
// products). A tile is one of
//   stats  logits of 256 packed rows and classes; a row's maximum and sum of exponentials of each
//          128 classes are kept, and the logits of its targets
//   G      the same logits again, turned into the loss's gradient (bf16) of a piece of the classes
//   dH     G W over classes of a piece: fp32 sums, added to those of the pieces before
//   dW     G^T H over the rows: a piece of the head's gradient
// The forward pass is one launch of stats tiles. The backward pass takes the classes in pieces: launch j
// holds the G tiles of piece j and the dH and dW tiles of piece j - 1, so that a launch has tiles enough
// to fill the machine and its last wave is a small part of it; two buffers of G take turns. Every sum
// has one order: results are the same in every run.
// Operands lie as they are: rows x features, classes x features and rows x classes are read
// K-major or MN-major (64 of M or N a 128-byte line), by descriptor, from the same TMA boxes of 64 x 64.
// G is rounded to bf16 because the tensor cores take it so; rows' weights enter it as shares of the largest one,
// so that equal weights leave its roundings independent (a common factor of 1 / 3580 rounded every target's
// entry the same way: gradients 2.8e-3 off, now 1.9e-3), and the gradients that it enters are rounded to bf16 as well.
//
// fp32: every operand is three bf16 numbers whose sum it is (8 bits each, next_parts), and a product of two is six of their nine
// products, the least first, in the same accumulators; the three that are left out are below 2^-24 of it.
//
// The tensor cores cut what an addition loses instead of rounding it, so a sum of many steps drifts towards zero: 320 steps
// of 16 k were 1e-5 of a logit off, which its exponential multiplies (fp32 gradients 5e-5). Where fp32 results come
// of it (logits, all fp32 products) a tile's k are cut in chunks of at most 32 steps (fp32: 16, each of
// which holds its six products), whose accumulators the epilogue's threads add up in registers, rounding, while the next
// chunk is multiplied. Chunks of 32, 16 and 8 steps: 700 fp32 rows of 512 features, 50304 classes, head gradient 1.2e-6, 7e-7 and
// 5e-7 off; loss and gradients of 645 such rows 671, 674 and 694 us. bf16, 64, 32 and 16 steps: losses of 400 rows of 5120 features 6e-7,
// 3e-7 and 2e-7 off; of 3331 rows of the Pythia-1.4B head 362, 378 and 415 us.
// The tensor cores bound it: 4096 bf16 rows, 32768 classes of 3584: stats 473 us (2.03 PFLOP/s), G 504, dH and dW 1017 (1.89
// PFLOP/s), the pipe 87 to 92% active. 768 fp32 rows, 50304 classes of 512: 124, 148 and 312 us (320 to 255 TFLOP/s of fp32 products, the pipe 87,
// 72 and 68% active: epilogues of short sums).
//   warp 0     TMA: A and B tiles of 64 k, 6 stages of 32 KB (both CTAs)
//   warp 1     TMEM, MMA issue (one thread of the even CTA)
//   warps 2-9  epilogue (two per TMEM lane quarter, 128 columns each)
// Every wait is bounded in time (device error word on give-up).
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "head.cuh"

namespace adadsf {
namespace {

constexpr int kHtTile = 256;                       // rows and columns of a pair's tile
constexpr int kHtK = 64;
constexpr int kHtStages = 6;
constexpr int kHtBox = 64 * 64 * 2;                // bytes of a TMA box
constexpr int kHtOperand = 2 * kHtBox;             // a CTA's 128 rows (or columns) of an operand
constexpr int kHtStage = 2 * kHtOperand;
constexpr int kHtEpiWarps = 8;
constexpr int kHtThreads = 64 + 32 * kHtEpiWarps;
constexpr int kHtBars = 2 * kHtStages + 5;
constexpr int kHtOut = 32 * 128;                   // an epilogue warp's 32 rows of 128 bytes on their way out
constexpr int kHtSmem = 1024 + kHtStages * kHtStage + kHtEpiWarps * kHtOut + kHtBars * 8 + 16;
constexpr uint32_t kHtDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;   // groups of 8 lines 1024 bytes apart, 128-byte swizzle

enum { kStats = 0, kG = 1, kDH = 2, kDW = 3 };

struct HtDev {
  const int32_t* count;      // packed rows
  const int32_t* rows;       // their rows
  int n;                     // rows
  int64_t cap;               // rows of the packed buffers, and of G
  int d, V, Vp;              // Vp: rows of a part of the head
  float inv_t;
  const int32_t* cls;        // targets by row, [k]
  const float* p;            // their weights (null: 1)
  int k;
  // stats
  float2* rec;               // [128 classes][cap]
  float* picked;             // [row][k]
  // gradients
  const float* lse;          // by row
  const float* g;            // by row (null: 1)
  const float* g_ref;        // the largest
  float temp;
  int v_g, n_g;              // G tiles: first class, class tiles (0: none)
  int v_d, kb_d;             // dH and dW: first class of the piece, its blocks of 64 classes (0: none)
  int splits, want_h, want_w, first, add_w;
  int ld_g;
  bf16* G;                   // the piece of the G tiles
  void* dh;                  // where a row's gradient is one sum; else null and its parts go to
  float* acc;                // [splits][cap][d]
  void* dw;
  int* err;
  unsigned long long timeout_ns;
};

struct Tile {
  int kind, mb, nb, kb0, nkb, slot;
};

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Tiles of a launch for `count` packed rows: dH, then dW, then G (or stats alone).
template <bool GRAD>
struct Tiles {
  int mbs, nbd, vt, n_h, n_w, n;
  __device__ Tiles(const HtDev& p, int count) {
    mbs = ceil_div(count, kHtTile);
    if (!GRAD) {
      vt = ceil_div(p.V, kHtTile);
      n_h = n_w = nbd = 0;
      n = mbs * vt;
      return;
    }
    nbd = ceil_div(p.d, kHtTile);
    vt = ceil_div(p.kb_d * kHtK, kHtTile);
    n_h = p.want_h && p.kb_d > 0 ? mbs * nbd * p.splits : 0;
    n_w = p.want_w ? vt * nbd : 0;
    n = n_h + n_w + mbs * p.n_g;
  }
  // Row tiles in groups, a group's packed rows in the L2 while the classes pass by.
  __device__ void by_class(int t, int classes, int* mb, int* nb) const {
    constexpr int kGroup = 16;
    const int per = kGroup * classes, g = t / per, in = t - g * per;
    const int rows = min(kGroup, mbs - g * kGroup);
    *nb = in / rows;
    *mb = g * kGroup + in % rows;
  }
  __device__ Tile at(const HtDev& p, int count, int t) const {
    Tile ti;
    ti.slot = ti.kb0 = 0;
    if (!GRAD) {
      ti.kind = kStats;
      ti.nkb = ceil_div(p.d, kHtK);
      by_class(t, vt, &ti.mb, &ti.nb);
      return ti;
    }
    if (t < n_h) {
      ti.kind = kDH;
      ti.mb = t % mbs;
      const int r = t / mbs;
      ti.nb = r % nbd;
      ti.slot = r / nbd;
      ti.kb0 = (int)((int64_t)p.kb_d * ti.slot / p.splits);
      ti.nkb = (int)((int64_t)p.kb_d * (ti.slot + 1) / p.splits) - ti.kb0;
      return ti;
    }
    t -= n_h;
    if (t < n_w) {
      ti.kind = kDW;
      ti.nb = t % nbd;
      ti.mb = t / nbd;
      ti.nkb = ceil_div(count, kHtK);
      return ti;
    }
    t -= n_w;
    ti.kind = kG;
    ti.nkb = ceil_div(p.d, kHtK);
    by_class(t, p.n_g, &ti.mb, &ti.nb);
    return ti;
  }
};

__device__ __forceinline__ uint64_t desc_of(uint32_t low) { return (uint64_t)kHtDescHigh << 32 | low; }

// 16-byte pieces of a warp's 32 rows of 128 bytes, swizzled so that neither side meets a bank twice.
__device__ __forceinline__ uint32_t out_at(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }

__device__ __forceinline__ void red_add4(float* p, const float4& v) {
  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// Blocks of 64 k whose products share an accumulator. G's logits are added up as those of the forward pass are, so that both passes
// have the same ones: q - 1 of a target of nearly all the weight is a difference of the two, and of one chain of 320
// steps beside chunks of 32 it was 6e-4 off where it is 3e-4 itself. bf16 gradients: sums of more than 65536 rows (or
// classes) are cut, below which the loss does not show: one of 4 million rows was 3.6e-3 short (head gradients 4.4e-3 off, of
// which roundings are 1.8e-3). Without the chunks of G's logits gradients of 27 rows at a 151936 x 1536 head took 338 us (346 with them), of
// 3330 at the Pythia-1.4B head 1361 (1412), of 3450 at the Qwen2.5-7B head 6950 (7090).
constexpr int kHtLong = 1024;
template <bool F32>
__device__ __forceinline__ int chunk_blocks(int kind) { return F32 ? kHeadChunkF32 : kind == kStats || kind == kG ? kHeadChunk : kHtLong; }

// A warp's loads from TMEM are done (tcgen05.wait::ld): only that is told, so the arrival is relaxed. Released, it waits
// until the warp's stores to global memory are performed (gradients of 500 tokens at the Qwen2.5-7B head 1104 -> 1079 us).
__device__ __forceinline__ void arrive_read(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

// A warp's 32 staged rows of 64 bf16 (swizzled as out_at does) to a matrix of global memory, which cuts them at its edges. The
// stage is free again after out_free(). Stored by the threads themselves: gradients of 27 tokens at a 151936 x 1536
// head 372 us, so 342; of 128 tokens 355, so 324; no difference with many rows.
__device__ __forceinline__ void out_store(const CUtensorMap& tm, const uint8_t* out, int col, int row, int lane) {
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(reinterpret_cast<uint64_t>(&tm)),
                 "r"(col), "r"(row), "r"(smem_u32(out))
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}
__device__ __forceinline__ void out_free(int lane) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  __syncwarp();
}

struct Walk {   // a row's targets, from the first one at or past the tile's first class
  const int32_t* cls;
  int j, k, next;
  __device__ __forceinline__ void start(const int32_t* c, int n, int c0, bool live) {
    cls = c;
    k = n;
    j = live ? first_class(c, n, c0) : n;
    next = j < k ? cls[j] : INT_MAX;
  }
  __device__ __forceinline__ void step() { next = ++j < k ? cls[j] : INT_MAX; }
};

__device__ __forceinline__ void stats_tile(const HtDev& p, const Tile& ti, int m, int half, bool live, uint32_t tacc, Walk& w) {
  constexpr float kLog2e = 1.4426950408889634f;
  const float c = p.inv_t * kLog2e;
  const int c0 = ti.nb * kHtTile + half * 128;
  float top = -INFINITY, sum = 0.f;
  const int64_t row = live ? p.rows[m] : 0;
#pragma unroll 1
  for (int ch = 0; ch < 4; ++ch) {
    const int cb = c0 + ch * 32;
    if (cb >= p.V) break;
    uint32_t r[32];
    tmem_ld32(tacc + ch * 32, r);
    tmem_ld_wait();
    if (cb + 32 > p.V) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (cb + i >= p.V) r[i] = 0xff800000u;   // no class: -inf
    }
    while (__any_sync(0xffffffffu, w.next < cb + 32)) {
      const float v = pick32(r, (w.next - cb) & 31);
      if (w.next < cb + 32) {
        p.picked[row * p.k + w.j] = v;
        w.step();
      }
    }
    float a = -INFINITY, b = -INFINITY;
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      a = fmax3(a, __uint_as_float(r[i]), __uint_as_float(r[i + 1]));
      b = fmax3(b, __uint_as_float(r[i + 2]), __uint_as_float(r[i + 3]));
    }
    const float now = fmax3(a, b, top);
    if (now > top) {
      sum *= top == -INFINITY ? 0.f : ex2_approx((top - now) * c);
      top = now;
    }
    // NaN logits leave the maximum but reach the sum; a maximum of -inf subtracts nothing
    const float base = top == -INFINITY ? 0.f : top;
    const float2 nb2 = make_float2(-base, -base), c2 = make_float2(c, c);
    float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      const float2 x = __fmul2_rn(__fadd2_rn(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), nb2), c2);
      const float2 y = __fmul2_rn(__fadd2_rn(make_float2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3])), nb2), c2);
      s0 = __fadd2_rn(s0, make_float2(ex2_approx(x.x), ex2_approx(x.y)));
      s1 = __fadd2_rn(s1, make_float2(ex2_approx(y.x), ex2_approx(y.y)));
    }
    sum += (s0.x + s0.y) + (s1.x + s1.y);
  }
  if (live) p.rec[(int64_t)(ti.nb * 2 + half) * p.cap + m] = make_float2(top, sum);
}

template <bool F32>
__device__ __forceinline__ void g_tile(const HtDev& p, const CUtensorMap& tm, const Tile& ti, int m, int half, bool live, uint32_t tacc,
                                       Walk& w, uint8_t* out, int lane) {
  constexpr float kLog2e = 1.4426950408889634f;
  const int64_t row = live ? p.rows[m] : 0;
  const float lse = live ? p.lse[row] : 0.f;
  const float g = live ? (p.g ? p.g[row] : 1.f) / *p.g_ref : 0.f;
  const float2 it2 = make_float2(p.inv_t, p.inv_t), ml2 = make_float2(-lse, -lse), e2 = make_float2(kLog2e, kLog2e);
  const float2 g2 = make_float2(g, g);
  const int m0 = m - lane;
  bf16* dst = p.G + (int64_t)m0 * p.ld_g + ti.nb * kHtTile + half * 128;
#pragma unroll 1
  for (int c32 = 0; c32 < 4; ++c32) {
    const int cb = p.v_g + ti.nb * kHtTile + half * 128 + c32 * 32;
    uint32_t r[32];
    tmem_ld32(tacc + c32 * 32, r);
    tmem_ld_wait();
    const bool edge = cb + 32 > p.V;
    float f[32];
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const float2 z = __ffma2_rn(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), it2, ml2);
      const float2 t = __fmul2_rn(z, e2);
      const float2 v = __fmul2_rn(make_float2(ex2_approx(t.x), ex2_approx(t.y)), g2);
      f[i] = v.x;
      f[i + 1] = v.y;
    }
    if (edge || !live) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (!live || cb + i >= p.V) f[i] = 0.f;
    }
    if (!F32) {
      if (!(c32 & 1)) out_free(lane);
#pragma unroll
      for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4*>(out + out_at(lane, (c32 & 1) * 4 + q)) = pack16(f + 8 * q, bf16());
    }
    while (__any_sync(0xffffffffu, w.next < cb + 32)) {
      const int at = (w.next - cb) & 31;
      const float l = pick32(r, at);
      if (w.next < cb + 32) {
        const int c = w.next;
        float want = 0.f;
        do {   // the same class twice: both weights
          want += p.p ? p.p[row * p.k + w.j] : 1.f;
          w.step();
        } while (w.next == c);
        const float v = (ex2_approx(fmaf(l, p.inv_t, -lse) * kLog2e) - want) * g;
        if (F32) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i == at) f[i] = v;
        } else {
          *reinterpret_cast<bf16*>(out + out_at(lane, (c32 & 1) * 4 + (at >> 3)) + (at & 7) * 2) = __float2bfloat16_rn(v);
        }
      }
    }
    if (F32) {
#pragma unroll 1
      for (int part = 0; part < 3; ++part) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = next_parts(f[8 * q + 2 * i], f[8 * q + 2 * i + 1]);
          }
          *reinterpret_cast<uint4*>(out + out_at(lane, q)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int rr = i * 8 + (lane >> 2), piece = lane & 3;
          const uint4 v = *reinterpret_cast<const uint4*>(out + out_at(rr, piece));
          *reinterpret_cast<uint4*>(dst + (part * p.cap + rr) * p.ld_g + c32 * 32 + piece * 8) = v;
        }
        __syncwarp();
      }
    } else if (c32 & 1) {
      out_store(tm, out, ti.nb * kHtTile + half * 128 + (c32 - 1) * 32, m0, lane);
    }
  }
}

template <bool F32>
__device__ __forceinline__ void dh_tile(const HtDev& p, const Tile& ti, int m0, int count, int half, uint32_t tacc, uint8_t* out,
                                        int lane) {
  const int c0 = ti.nb * kHtTile + half * 128;
  if (!F32) out_free(lane);
  if (p.dh) {   // all classes in one sum: no partial sums to be joined
    using T = typename std::conditional<F32, float, bf16>::type;
    constexpr int V = Elem<T>::kVec, COLS = 8 * V;
    const float scale = *p.g_ref * p.temp;
    const int64_t row = m0 + lane < count ? p.rows[m0 + lane] : -1;
#pragma unroll 1
    for (int c = 0; c < 128; c += COLS) {
      if (c0 + c >= p.d) break;
#pragma unroll
      for (int h = 0; h < COLS; h += 32) {
        uint32_t r[32];
        tmem_ld32(tacc + c + h, r);
        tmem_ld_wait();
#pragma unroll
        for (int q = 0; q < 32 / V; ++q) {
          float f[V];
#pragma unroll
          for (int i = 0; i < V; ++i) f[i] = __uint_as_float(r[V * q + i]) * scale;
          *reinterpret_cast<uint4*>(out + out_at(lane, h / V + q)) = pack16(f, T());
        }
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int rr = i * 4 + (lane >> 3), piece = lane & 7;
        const uint4 v = *reinterpret_cast<const uint4*>(out + out_at(rr, piece));
        const int64_t to = __shfl_sync(0xffffffffu, row, rr);
        if (to >= 0 && c0 + c + piece * V < p.d)
          *reinterpret_cast<uint4*>(static_cast<T*>(p.dh) + to * p.d + c0 + c + piece * V) = v;
      }
      __syncwarp();
    }
    return;
  }
  float* dst = p.acc + ((int64_t)ti.slot * p.cap + m0) * p.d + c0;
#pragma unroll 1
  for (int ch = 0; ch < 4; ++ch) {
    if (c0 + ch * 32 >= p.d) break;
    uint32_t r[32];
    tmem_ld32(tacc + ch * 32, r);
    tmem_ld_wait();
#pragma unroll
    for (int q = 0; q < 8; ++q)
      *reinterpret_cast<uint4*>(out + out_at(lane, q)) =
          ti.nkb ? make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]) : make_uint4(0, 0, 0, 0);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int rr = i * 4 + (lane >> 3), piece = lane & 7;
      const float4 v = *reinterpret_cast<const float4*>(out + out_at(rr, piece));
      float* at = dst + (int64_t)rr * p.d + ch * 32 + piece * 4;
      if (m0 + rr < count && c0 + ch * 32 + piece * 4 < p.d) {
        if (p.first) *reinterpret_cast<float4*>(at) = v;
        else red_add4(at, v);
      }
    }
    __syncwarp();
  }
}

// 32 columns of the accumulator as this thread's part of the head's gradient, in vectors.
template <typename T>
__device__ __forceinline__ void dw_columns(const HtDev& p, const Tile& ti, uint32_t tacc, float scale, const T* old_row, bool in_row,
                                           int cols, uint4* held) {
  constexpr int V = Elem<T>::kVec;
  uint32_t r[32];
  tmem_ld32(tacc, r);
  tmem_ld_wait();
#pragma unroll
  for (int q = 0; q < 32 / V; ++q) {
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = ti.nkb ? __uint_as_float(r[V * q + i]) * scale : 0.f;
    if (p.add_w && in_row && q * V < cols) {   // what is there is added before the one rounding
      float old[V];
      load_vec(old_row + q * V, old);
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] += old[i];
    }
    held[q] = pack16(f, T());
  }
}

// Rows of the head's gradient. bf16: the accumulator is free again (release) before the stores: with few rows a
// tile has one block of products, and its stores are what there is to do. (fp32 has no registers for that.)
template <bool F32, typename Release>
__device__ __forceinline__ void dw_tile(const HtDev& p, const CUtensorMap& tm, const Tile& ti, int v0, int half, uint32_t tacc,
                                        uint8_t* out, int lane, Release release) {
  using T = typename std::conditional<F32, float, bf16>::type;
  constexpr int V = Elem<T>::kVec, COLS = 8 * V;   // columns of 128 bytes
  const float scale = *p.g_ref * p.temp;
  const int c0 = ti.nb * kHtTile + half * 128;
  T* dst = static_cast<T*>(p.dw) + (int64_t)v0 * p.d + c0;
  const bool in_row = v0 + lane < p.V;
  uint4 held[F32 ? 8 : 16];
  if (!F32) {
#pragma unroll
    for (int c = 0; c < 128; c += 32)
      dw_columns<T>(p, ti, tacc + c, scale, dst + (int64_t)lane * p.d + c, in_row, p.d - c0 - c, held + (F32 ? 0 : c / V));
    release();
  }
#pragma unroll
  for (int c = 0; c < 128; c += COLS) {
    if (c0 + c >= p.d) break;
    if (F32) dw_columns<T>(p, ti, tacc + c, scale, dst + (int64_t)lane * p.d + c, in_row, p.d - c0 - c, held);
    if (!F32) out_free(lane);
#pragma unroll
    for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(out + out_at(lane, q)) = held[F32 ? q : c / V + q];
    if (!F32) {
      if (v0 < p.V) out_store(tm, out, c0 + c, v0, lane);
      continue;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int rr = i * 4 + (lane >> 3), piece = lane & 7;
      const uint4 v = *reinterpret_cast<const uint4*>(out + out_at(rr, piece));
      if (v0 + rr < p.V && c0 + c + piece * V < p.d) *reinterpret_cast<uint4*>(dst + (int64_t)rr * p.d + c + piece * V) = v;
    }
    __syncwarp();
  }
  if (F32) release();
}

template <bool GRAD, bool F32>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kHtThreads, 1)
    head_tc_kernel(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                   const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmGo,
                   const __grid_constant__ CUtensorMap tmDw, const __grid_constant__ HtDev p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t ring = smem_u32(smem);
  uint8_t* outs = smem + kHtStages * kHtStage;
  uint64_t* bars = reinterpret_cast<uint64_t*>(outs + kHtEpiWarps * kHtOut);
  const uint32_t full0 = smem_u32(bars);
  const uint32_t empty0 = full0 + 8 * kHtStages;
  const uint32_t tfull0 = empty0 + 8 * kHtStages;
  const uint32_t tempty0 = tfull0 + 16;
  const uint32_t drain = tempty0 + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kHtBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1;
  const int num_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kHtStages; ++s) {
      mbar_init(full0 + 8 * s, 1);   // the even CTA's producer arms both CTAs' bytes
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(tfull0 + 8 * a, 1);
      mbar_init(tempty0 + 8 * a, 2 * kHtEpiWarps);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tmP);
    if (!F32) tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmW);
    if (GRAD) tma_prefetch_desc(&tmG);
    if (GRAD && !F32) {
      tma_prefetch_desc(&tmGo);
      tma_prefetch_desc(&tmDw);
    }
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), 512);
  __syncwarp();
  tc_fence_before();
  cluster_sync();   // both CTAs' barriers initialised, TMEM allocated
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t full_lead = map_to_cta(full0, 0);
  const uint32_t tempty_lead = map_to_cta(tempty0, 0);
  pdl_wait();
  const int count = *p.count;
  const CUtensorMap& tmH = !F32 && count == p.n ? tmA : tmP;   // bf16 rows that all count were not packed
  const Tiles<GRAD> tiles(p, count);
  constexpr int TERMS = F32 ? kHeadTerms : 1;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (both CTAs)
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      int64_t issued = 0;
      bool ok = true;
      for (int t = pair; t < tiles.n && ok; t += num_pairs) {
        const Tile ti = tiles.at(p, count, t);
        const int a0 = ti.mb * kHtTile + (int)rank * 128, b0 = ti.nb * kHtTile + (int)rank * 128;
        const int chunk = chunk_blocks<F32>(ti.kind);
        int first = 0, kb = 0, term = 0;   // of the chunk, in it, and the product of parts
        int64_t pa = 0, pb = 0;            // rows before the parts
        auto parts = [&] {
          if (!F32) return;
          pa = head_part_a(term) * p.cap;
          pb = head_part_b(term) * (!GRAD || ti.kind != kDW ? (int64_t)p.Vp : p.cap);
        };
        parts();
        for (int i = ti.nkb * TERMS; i > 0; --i) {
          if (!mbar_wait_bounded(empty0 + 8 * stage, phase ^ 1, abort_flag, p.err, p.timeout_ns)) {
            ok = false;
            break;
          }
          const uint32_t fb = full_lead + 8 * stage, a_s = ring + stage * kHtStage, b_s = a_s + kHtOperand;
          if (rank == 0) mbar_arrive_expect_tx(full0 + 8 * stage, 2 * kHtStage);
          const int k0 = (ti.kb0 + first + kb) * kHtK;
          if (!GRAD || ti.kind == kG) {   // H and W, both K-major: boxes of 64 rows
            const int a = (int)(a0 + pa), b = (int)((GRAD ? p.v_g : 0) + b0 + pb);
            tma_load_2d_pair(a_s, &tmH, k0, a, fb);
            tma_load_2d_pair(a_s + kHtBox, &tmH, k0, a + 64, fb);
            tma_load_2d_pair(b_s, &tmW, k0, b, fb);
            tma_load_2d_pair(b_s + kHtBox, &tmW, k0, b + 64, fb);
          } else if (ti.kind == kDH) {    // G K-major, W as it lies (N = features)
            const int a = (int)(a0 + pa), b = (int)(p.v_d + k0 + pb);
            tma_load_2d_pair(a_s, &tmG, k0, a, fb);
            tma_load_2d_pair(a_s + kHtBox, &tmG, k0, a + 64, fb);
            tma_load_2d_pair(b_s, &tmW, b0, b, fb);
            tma_load_2d_pair(b_s + kHtBox, &tmW, b0 + 64, b, fb);
          } else {                        // both as they lie (M = classes, N = features, K = rows)
            const int a = (int)(k0 + pa), b = (int)(k0 + pb);
            tma_load_2d_pair(a_s, &tmG, a0, a, fb);
            tma_load_2d_pair(a_s + kHtBox, &tmG, a0 + 64, a, fb);
            tma_load_2d_pair(b_s, &tmH, b0, b, fb);
            tma_load_2d_pair(b_s + kHtBox, &tmH, b0 + 64, b, fb);
          }
          if (++kb == min(chunk, ti.nkb - first)) {
            kb = 0;
            if (++term == TERMS) {
              term = 0;
              first += chunk;
            }
            parts();
          }
          ++issued;
          if (++stage == kHtStages) { stage = 0; phase ^= 1; }
        }
      }
      pdl_trigger();
      if (rank == 0) {   // drain: the copies issued last (both CTAs') have landed
        for (int s = 0; s < kHtStages; ++s) {
          if (issued <= s) break;
          const int64_t last = s + ((issued - 1 - s) / kHtStages) * kHtStages;
          mbar_wait_drain(full0 + 8 * s, (uint32_t)((last / kHtStages) & 1), p.timeout_ns);
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (even CTA)
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = idesc_bf16_f32(kHtTile, kHtTile);
      constexpr uint32_t kMajorK = 1u << 16, kMajorMN = (uint32_t)(kHtBox >> 4) << 16;   // next 64 of M or N
      int stage = 0;
      uint32_t phase = 0;
      int it = 0;
      bool ok = true;
      for (int t = pair; t < tiles.n && ok; t += num_pairs) {
        const Tile ti = tiles.at(p, count, t);
        const bool a_mn = GRAD && ti.kind == kDW, b_mn = GRAD && (ti.kind == kDW || ti.kind == kDH);
        const uint32_t id = idesc | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
        const uint32_t a_hi = a_mn ? kMajorMN : kMajorK, b_hi = b_mn ? kMajorMN : kMajorK;
        const uint32_t a_step = a_mn ? 128 : 2, b_step = b_mn ? 128 : 2;   // 16 k on, in 16 bytes
        const int chunk = chunk_blocks<F32>(ti.kind);
        int first = 0;
        do {   // a chunk (one without blocks where there is no k)
          const int acc = it & 1, blocks = min(chunk, ti.nkb - first) * TERMS;
          if (!mbar_wait_bounded(tempty0 + 8 * acc, ((it >> 1) & 1) ^ 1, abort_flag, p.err, p.timeout_ns)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + acc * 256;
          for (int kb = 0; kb < blocks; ++kb) {
            if (!mbar_wait_bounded(full0 + 8 * stage, phase, abort_flag, p.err, p.timeout_ns)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t a_s = ring + stage * kHtStage;
            const uint32_t a_lo = ((a_s & 0x3FFFFu) >> 4) | a_hi, b_lo = (((a_s + kHtOperand) & 0x3FFFFu) >> 4) | b_hi;
#pragma unroll
            for (int k = 0; k < kHtK / 16; ++k)
              tc_mma_f16_pair(d_tmem, desc_of(a_lo + k * a_step), desc_of(b_lo + k * b_step), id, (kb > 0 || k > 0) ? 1u : 0u);
            tc_commit_pair_multicast(empty0 + 8 * stage, 0x3);   // both CTAs' stage free
            if (++stage == kHtStages) { stage = 0; phase ^= 1; }
          }
          if (!ok) break;
          tc_commit_pair_multicast(tfull0 + 8 * acc, 0x3);   // both CTAs' accumulators ready
          ++it;
          first += chunk;
        } while (first < ti.nkb);
      }
      tc_commit_pair_multicast(drain, 0x1);
      mbar_wait_drain(drain, 0, p.timeout_ns);
    }
  } else {
    // ------------------------------------------------------------ epilogue (warps 2..9, both CTAs)
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint8_t* out = outs + (warp - 2) * kHtOut;
    int it = 0;
    bool ok = true;
    for (int t = pair; t < tiles.n && ok; t += num_pairs) {
      const Tile ti = tiles.at(p, count, t);
      const int m0 = ti.mb * kHtTile + (int)rank * 128 + quarter * 32, m = m0 + lane;
      Walk w;
      if (!GRAD || ti.kind == kG) {   // the row's targets are found under the tile's products
        const bool live = m < count;
        w.start(p.cls + (live ? (int64_t)p.rows[m] * p.k : 0), p.k, (GRAD ? p.v_g : 0) + ti.nb * kHtTile + half * 128, live);
      }
      const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16) + half * 128;
      auto wait = [&] {
        int got = 0;
        if (lane == 0) got = mbar_wait_bounded(tfull0 + 8 * (it & 1), (it >> 1) & 1, abort_flag, p.err, p.timeout_ns);
        ok = __shfl_sync(0xffffffffu, got, 0) != 0;
        tc_fence_after();
      };
      auto release = [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_read(tempty_lead + 8 * (it & 1));
        ++it;
      };
      wait();
      if (!ok) break;
      const int chunk = chunk_blocks<F32>(ti.kind);
      if (ti.nkb > chunk) {
        float run[128];
        int first = chunk;
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          uint32_t r[32];
          tmem_ld32(lanes + (it & 1) * 256 + c, r);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i) run[c + i] = __uint_as_float(r[i]);
        }
        release();
        for (;;) {
          wait();
          if (!ok) break;
          first += chunk;
          const bool last = first >= ti.nkb;
#pragma unroll
          for (int c = 0; c < 128; c += 16) {
            uint32_t r[16];
            tmem_ld8(lanes + (it & 1) * 256 + c, r);
            tmem_ld8(lanes + (it & 1) * 256 + c + 8, r + 8);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              run[c + i] += __uint_as_float(r[i]);
              r[i] = __float_as_uint(run[c + i]);
            }
            if (last) tmem_st16(lanes + (it & 1) * 256 + c, r);   // where the tile's epilogue finds them
          }
          if (last) break;
          release();
        }
        if (!ok) break;
        tmem_st_wait();
      }
      const uint32_t tacc = lanes + (it & 1) * 256;
      if (!GRAD) stats_tile(p, ti, m, half, m < count, tacc, w);
      else if (ti.kind == kG) g_tile<F32>(p, tmGo, ti, m, half, m < count, tacc, w, out, lane);
      else if (ti.kind == kDH) dh_tile<F32>(p, ti, m0, count, half, tacc, out, lane);
      else dw_tile<F32>(p, tmDw, ti, p.v_d + m0, half, tacc, out, lane, release);
      if (!GRAD || ti.kind != kDW) release();
    }
    if (GRAD && !F32 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // this warp's stores are done
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();   // the pair's MMAs and copies are done before TMEM and smem go
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

bool head_maps(bool f32, const Head& a, CUtensorMap* th, CUtensorMap* tw) {
  const uint64_t parts = f32 ? 3 : 1, ld = (uint64_t)a.ld;
  return make_tmap_bf16(th, a.packed, parts * (uint64_t)a.cap, ld, ld, 64, 64) &&
         make_tmap_bf16(tw, f32 ? a.w_parts : a.w, f32 ? parts * (uint64_t)a.Vp : (uint64_t)a.V, ld, ld, 64, 64);
}

HtDev head_dev(const Head& a, const Dev& dev) {
  HtDev p = {};
  p.count = a.count;
  p.rows = a.rows;
  p.n = (int)a.n;
  p.cap = a.cap;
  p.d = a.d;
  p.V = a.V;
  p.Vp = a.Vp;
  p.inv_t = 1.f / a.temp;
  p.temp = a.temp;
  p.cls = a.cls;
  p.p = a.p;
  p.k = a.k;
  p.rec = a.rec;
  p.picked = a.picked;
  p.lse = a.lse;
  p.g = a.g;
  p.g_ref = a.g_ref;
  p.err = dev.err;
  p.timeout_ns = kWaitTimeoutNs;
  return p;
}

int ceil_to(int64_t a, int b) { return (int)((a + b - 1) / b); }

template <bool GRAD, bool F32>
cudaError_t launch_tiles(int64_t tiles, const Head& a, const CUtensorMap& tg, const CUtensorMap& tgo, const CUtensorMap& tdw,
                         const HtDev& p, const Dev& dev) {
  const cudaError_t e = allow_smem<head_tc_kernel<GRAD, F32>, kHtSmem>();
  if (e != cudaSuccess || tiles == 0) return e;
  CUtensorMap th, ta = {}, tw;
  if (!head_maps(F32, a, &th, &tw)) return cudaErrorInvalidValue;
  if (!F32 && !make_tmap_bf16(&ta, a.h, (uint64_t)a.n, (uint64_t)a.d, (uint64_t)a.d, 64, 64)) return cudaErrorInvalidValue;
  const int pairs = (int)std::min<int64_t>(tiles, dev.num_sms / 2);
  return launch_pdl(head_tc_kernel<GRAD, F32>, dim3(2 * pairs), dim3(kHtThreads), kHtSmem, dev.stream, th, ta, tw, tg, tgo, tdw,
                    p);
}

}  // namespace

cudaError_t head_stats(int dtype, const Head& a, const Dev& dev) {
  const int64_t tiles = (int64_t)ceil_to(a.n, kHtTile) * ceil_to(a.V, kHtTile);
  const CUtensorMap none = {};
  return dtype == kBF16 ? launch_tiles<false, false>(tiles, a, none, none, none, head_dev(a, dev), dev)
                        : launch_tiles<false, true>(tiles, a, none, none, none, head_dev(a, dev), dev);
}

cudaError_t head_grad(int dtype, const Head& a, int buf, int64_t v_g, int n_g, int64_t v_d, int n_d, bool first, const Dev& dev) {
  CUtensorMap tg, tgo = {}, tdw = {};
  if (dtype == kBF16 &&
      (!make_tmap_bf16(&tgo, a.G[buf], (uint64_t)a.cap, (uint64_t)a.piece, (uint64_t)a.piece, 64, 32) ||
       (a.dw && !make_tmap_bf16(&tdw, a.dw, (uint64_t)a.V, (uint64_t)a.d, (uint64_t)a.d, 64, 32))))
    return cudaErrorInvalidValue;
  if (!make_tmap_bf16(&tg, a.G[buf ^ 1], (uint64_t)a.cap * (dtype == kBF16 ? 1 : 3), (uint64_t)a.piece, (uint64_t)a.piece, 64, 64))
    return cudaErrorInvalidValue;
  HtDev p = head_dev(a, dev);
  p.v_g = (int)v_g;
  p.n_g = ceil_to(n_g, kHtTile);
  p.v_d = (int)v_d;
  p.kb_d = ceil_to(n_d, kHtK);
  p.splits = a.splits;
  p.want_h = a.dh != nullptr;
  p.want_w = a.dw != nullptr;
  p.first = first;
  p.add_w = a.add_w;
  p.ld_g = a.piece;
  p.G = static_cast<bf16*>(a.G[buf]);
  p.dh = a.dh_whole ? a.dh : nullptr;
  p.acc = a.dh_acc;
  p.dw = a.dw;
  const int64_t mbs = ceil_to(a.n, kHtTile), nbd = ceil_to(a.d, kHtTile);
  const int64_t tiles = mbs * p.n_g + (p.want_h && n_d ? mbs * nbd * p.splits : 0) + (p.want_w ? ceil_to(n_d, kHtTile) * nbd : 0);
  if (dtype != kBF16) return launch_tiles<true, true>(tiles, a, tg, tgo, tdw, p, dev);
  return launch_tiles<true, false>(tiles, a, tg, tgo, tdw, p, dev);
}

}  // namespace adadsf
