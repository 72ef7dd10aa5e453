// The losses' forward pass for few rows (at most kHeadFewRows, fp32 kHeadFewRowsF32), and G of few fp32 rows from the same logits: what
// bounds them is reading the head once.
//
// The operands change places against head_tc.cu: 128 classes are the M of a product and the packed rows, up to
// 128 in steps of 16, its N, so that the tensor cores spend on a block of classes what its rows need (with 256 rows
// a tile, 24 rows took as long as 256). A CTA takes one range of
// classes, in units of 32, and keeps a running maximum and sum of exponentials a row: one record a CTA and row.
// fp32: the head's numbers are split into their three bf16 parts (see next_parts) on the way into shared
// memory, by warps that read them a block ahead; a pass of its own wrote and read again three times the head's bytes.
// The rows' parts lie one behind the other, so that w1 (h2, h3) and w2 (h1, h2) are one product each, beside w3 h1
// and w1 h1: four products a step in place of six. The large one, w1 h1, has columns of its own, since what an
// addition cuts off goes by the accumulator (see head_tc.cu, also for the chunks of k).
// Measured, a graph's pass: 24 tokens of the Pythia-160M head 24.2 us with packing and joining (its bytes: 11.4), 77 fp32 tokens of
// the Pythia-70M head 53.7 (15; chunks of 32 steps 52.4, at twice the error).
//   warp 0       TMA: the rows' blocks of 64 k (fp32: three parts), the head's blocks (bf16)
//   warp 1       TMEM, MMA issue (one thread), accumulators double-buffered
//   then 8 (fp32 12) warps, epilogue: four of them take 32 rows of a tile through shared memory, which turns classes
//                into columns
//   then 8 warps, fp32: the head's parts
// Every wait is bounded in time (device error word on give-up).
#include <cuda.h>

#include <algorithm>

#include "head.cuh"

namespace adadsf {
namespace {

constexpr int kHfM = 128;                        // classes of a tile
constexpr int kHfUnit = 32;                      // classes of a box
constexpr int kHfK = 64;
constexpr int kHfPart = kHfM * kHfK * 2;         // bytes of a block of classes (one part)
constexpr int kHfConvWarps = 8;
constexpr int kHfOutLd = kHfM + 4;               // floats of a staged row
constexpr int kHfOut = 32 * kHfOutLd * 4;        // 32 rows of a tile
constexpr int kHfMaxStages = 8;
constexpr int kHfBars = 2 * kHfMaxStages + 5;
constexpr uint32_t kHfDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;

template <bool F32>
struct HfCfg {
  static constexpr int PARTS = F32 ? 3 : 1;
  static constexpr int COLS = F32 ? 256 : 128;   // of an accumulator
  static constexpr int GROUPS = F32 ? 3 : 2;     // of four epilogue warps
  static constexpr int TURNS = F32 ? 1 : 2;      // times 32 rows that a group takes
  static constexpr int EPI = 4 * GROUPS;
  static constexpr int CHUNK = F32 ? kHeadChunkF32 : kHeadChunk;
  static constexpr int THREADS = 64 + 32 * (EPI + (F32 ? kHfConvWarps : 0));
  static constexpr int RING = F32 ? 2 * 3 * (kHfPart + kHeadFewRowsF32 * 128) : 196608;
  static constexpr int SMEM = 1024 + RING + GROUPS * kHfOut + kHfBars * 8 + 16;
  __host__ __device__ static int stage(int n) { return PARTS * (kHfPart + n * 128); }
  __host__ __device__ static int stages(int n) {
    const int s = RING / stage(n);
    return s < kHfMaxStages ? s : kHfMaxStages;
  }
  static_assert(32 * GROUPS * TURNS >= (F32 ? kHeadFewRowsF32 : kHeadFewRows), "rows");
  static_assert(PARTS * (F32 ? kHeadFewRowsF32 : kHeadFewRows) <= COLS, "columns");
};

struct HfDev {
  const int32_t *count, *rows;
  const float* w;            // fp32 head
  int64_t cap;
  int d, V, n, n_rows;       // n: rows, to a multiple of 16
  float inv_t;
  const int32_t* cls;
  int k;
  float2* rec;               // [CTA][cap]
  float* picked;
  int v0, v1;                // the classes: all of them, or a piece
  // G of a piece
  const float *pw, *lse, *g, *g_ref;   // weights of the targets [row][k]; by row
  bf16* G;                   // three parts of [cap][ld_g]
  int ld_g;
  int* err;
  unsigned long long timeout_ns;
};

// A product, and the arrival when all so far are done, issued by the lane with lead != 0 of a warp that comes along.
__device__ __forceinline__ void few_mma(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %6};\n\tmov.b64 db, {%2, %6};\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(lead), "r"(kHfDescHigh)
      : "memory");
}
__device__ __forceinline__ void few_commit(uint32_t bar, uint32_t lead) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(lead)
      : "memory");
}

// Whether ok holds in all 128 threads of a barrier.
__device__ __forceinline__ bool group_agrees(int id, bool ok) {
  int all;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\t"
      "bar.red.and.pred q, %1, 128, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(id), "r"((int)ok)
      : "memory");
  return all != 0;
}

// 32 classes of a row's gradient from its logits (staged), in three parts; zeros for a row behind the last one. Classes from c1 on
// are another CTA's.
__device__ __forceinline__ void g_vector(const HfDev& p, const float* l, int cb, int c1, int m, bool live) {
  constexpr float kLog2e = 1.4426950408889634f;
  if (cb >= c1) return;
  bf16* dst = p.G + (int64_t)m * p.ld_g + (cb - p.v0);
  const int64_t line = live ? (int64_t)p.rows[m] : 0;
  const float lse = live ? p.lse[line] : 0.f, g = live ? (p.g ? p.g[line] : 1.f) / *p.g_ref : 0.f;
  int j = live ? first_class(p.cls + line * p.k, p.k, cb) : p.k;
  int next = j < p.k ? p.cls[line * p.k + j] : INT_MAX;
#pragma unroll 1
  for (int b = 0; b < 32; b += 8) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = cb + b + i;
      float v = 0.f;
      if (live && c < p.V) {
        v = ex2_approx(fmaf(l[b + i], p.inv_t, -lse) * kLog2e);
        if (c == next) {
          float want = 0.f;
          do {   // the same class twice: both weights
            want += p.pw ? p.pw[line * p.k + j] : 1.f;
            next = ++j < p.k ? p.cls[line * p.k + j] : INT_MAX;
          } while (next == c);
          v -= want;
        }
        v *= g;
      }
      f[i] = v;
    }
#pragma unroll
    for (int part = 0; part < 3; ++part) {
      uint32_t u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = next_parts(f[2 * i], f[2 * i + 1]);
      *reinterpret_cast<uint4*>(dst + part * p.cap * p.ld_g + b) = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
}

template <bool F32, bool GRAD>
__global__ void __launch_bounds__(HfCfg<F32>::THREADS, 1)
    head_few_kernel(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                    const __grid_constant__ CUtensorMap tmW1, const __grid_constant__ HfDev p) {
  using C = HfCfg<F32>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t ring = smem_u32(smem);
  float* outs = reinterpret_cast<float*>(smem + C::RING);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::RING + C::GROUPS * kHfOut);
  const uint32_t full0 = smem_u32(bars);
  const uint32_t empty0 = full0 + 8 * kHfMaxStages;
  const uint32_t tfull0 = empty0 + 8 * kHfMaxStages;
  const uint32_t tempty0 = tfull0 + 16;
  const uint32_t drain = tempty0 + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kHfBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int stage_bytes = C::stage(p.n), stages = C::stages(p.n);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // this CTA's classes, in tiles of 128 of which the last may be short
  const int units = (p.v1 - p.v0 + kHfUnit - 1) / kHfUnit;
  const int c_begin = p.v0 + (int)((int64_t)units * blockIdx.x / gridDim.x) * kHfUnit;
  const int c_end = min(p.v1, p.v0 + (int)((int64_t)units * (blockIdx.x + 1) / gridDim.x) * kHfUnit);
  const int tiles = (c_end - c_begin + kHfM - 1) / kHfM, nkb = (p.d + kHfK - 1) / kHfK;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(full0 + 8 * s, 1 + (F32 ? kHfConvWarps : 0));
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(tfull0 + 8 * a, 1);
      mbar_init(tempty0 + 8 * a, C::EPI);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tmP);
    if (!F32) tma_prefetch_desc(&tmA);
    if (!F32) tma_prefetch_desc(&tmW);   // boxes of a whole tile; tmW1: of a unit
  }
  if (warp == 1) tmem_alloc(smem_u32(tmem_slot), 2 * C::COLS);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      int64_t issued = 0;
      bool ok = true;
      const int total = tiles * nkb;
      // bf16: the head's next block (weights: an earlier launch of this call waited for whatever wrote them)
      int c0 = c_begin, w_k = 0;
      auto head = [&](int s) {
        const uint32_t bar = full0 + 8 * s, to = ring + s * stage_bytes;
        const int classes = c_end - c0;
        if (classes >= kHfM) {
          mbar_arrive_expect_tx(bar, kHfPart + p.n * 128);
          tma_load_2d(to, &tmW, w_k, c0, bar);
        } else {
          const int boxes = (classes + kHfUnit - 1) / kHfUnit;
          mbar_arrive_expect_tx(bar, boxes * kHfUnit * 128 + p.n * 128);
          for (int b = 0; b < boxes; ++b) tma_load_2d(to + b * kHfUnit * 128, &tmW1, w_k, c0 + b * kHfUnit, bar);
        }
        w_k += kHfK;
        if (w_k >= p.d) {
          w_k = 0;
          c0 += kHfM;
        }
      };
      const int pre = F32 ? 0 : min(total, stages);
      for (int i = 0; i < pre; ++i) head(i);
      pdl_wait();
      const CUtensorMap& tmH = !F32 && *p.count == p.n_rows ? tmA : tmP;   // bf16 rows that all count were not packed
      int k = 0;
      for (int i = 0; i < total && ok; ++i) {
        if (i >= pre) {
          if (!mbar_wait_bounded(empty0 + 8 * stage, phase ^ 1, abort_flag, p.err, p.timeout_ns)) {
            ok = false;
            break;
          }
          if (F32) mbar_arrive_expect_tx(full0 + 8 * stage, 3 * p.n * 128);
          else head(stage);
        }
#pragma unroll
        for (int q = 0; q < C::PARTS; ++q)
          tma_load_2d(ring + stage * stage_bytes + C::PARTS * kHfPart + q * p.n * 128, &tmH, k, (int)(q * p.cap), full0 + 8 * stage);
        k += kHfK;
        if (k >= p.d) k = 0;
        ++issued;
        if (++stage == stages) { stage = 0; phase ^= 1; }
      }
      pdl_trigger();
      for (int s = 0; s < stages; ++s) {   // drain: the copies issued last have landed
        if (issued <= s) break;
        const int64_t last = s + ((issued - 1 - s) / stages) * stages;
        mbar_wait_drain(full0 + 8 * s, (uint32_t)((last / stages) & 1), p.timeout_ns);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    // all lanes come along, one of them issues: with warp-uniform operands a product takes no moves between
    // register files, which took longer than a product of few columns
    const uint32_t idesc = idesc_bf16_f32(kHfM, p.n), idesc2 = idesc_bf16_f32(kHfM, 2 * p.n), lead = lane == 0;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      int got = 0;
      if (lane == 0) got = mbar_wait_bounded(bar, parity, abort_flag, p.err, p.timeout_ns);
      return __shfl_sync(0xffffffffu, got, 0) != 0;
    };
    int it = 0;
    for (int tile = 0; tile < tiles && ok; ++tile) {
      for (int first = 0; first < nkb && ok; first += C::CHUNK, ++it) {
        const int acc = it & 1, blocks = min(C::CHUNK, nkb - first);
        if (!wait(tempty0 + 8 * acc, ((it >> 1) & 1) ^ 1)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t d = tmem_base + acc * C::COLS;
        for (int kb = 0; kb < blocks; ++kb) {
          if (!wait(full0 + 8 * stage, phase)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t w_s = ring + stage * stage_bytes, h_s = w_s + C::PARTS * kHfPart;
          const uint32_t w = (w_s & 0x3FFFFu) >> 4 | 1u << 16, h = (h_s & 0x3FFFFu) >> 4 | 1u << 16;
          const uint32_t w1 = kHfPart >> 4, h1 = p.n * 8;   // a part on, in 16 bytes
#pragma unroll
          for (int k = 0; k < 2 * kHfK / 16; k += 2) {
            const uint32_t more = kb > 0 || k > 0 ? 1u : 0u;
            if (F32) {
              few_mma(d + p.n, w + k, h + h1 + k, idesc2, more, lead);
              few_mma(d + p.n, w + w1 + k, h + k, idesc2, 1u, lead);
              few_mma(d + p.n, w + 2 * w1 + k, h + k, idesc, 1u, lead);
            }
            few_mma(d, w + k, h + k, idesc, more, lead);
          }
          few_commit(empty0 + 8 * stage, lead);
          if (++stage == stages) { stage = 0; phase ^= 1; }
        }
        if (ok) few_commit(tfull0 + 8 * acc, lead);
      }
    }
    few_commit(drain, lead);
    if (lane == 0) mbar_wait_drain(drain, 0, p.timeout_ns);
  } else if (warp < 2 + C::EPI) {
    // ------------------------------------------------------------ epilogue
    pdl_wait();
    const int count = *p.count;
    const int quarter = warp & 3, group = (warp - 2) >> 2;
    const int t = quarter * 32 + lane, r = t >> 2, q = t & 3;   // thread of the group; its row of 32, its quarter of the classes
    const float c = p.inv_t * 1.4426950408889634f;
    float* out = outs + group * (kHfOut / 4);
    float top[C::TURNS], sum[C::TURNS];
    int next[C::TURNS];
    const int chunks = (min(count, p.n) + 31) / 32;
    const int rows_zero = (count + kHeadZeroPad - 1) / kHeadZeroPad * kHeadZeroPad;   // G's rows past the last one are zero as far
#pragma unroll
    for (int u = 0; u < C::TURNS; ++u) {
      const int m = (group + C::GROUPS * u) * 32 + r;
      top[u] = -INFINITY;
      sum[u] = 0.f;
      next[u] = !GRAD && q == 0 && m < count ? first_class(p.cls + (int64_t)p.rows[m] * p.k, p.k, c_begin) : p.k;
    }
    bool ok = true;
    int it = 0;
    for (int tile = 0; tile < tiles && ok; ++tile) {
      const int c0 = c_begin + tile * kHfM, c1 = min(c_end, c0 + kHfM);
      float run[C::TURNS][32];
      for (int first = 0; first < nkb; first += C::CHUNK, ++it) {
        const int acc = it & 1;
        int got = 0;
        if (lane == 0) got = mbar_wait_bounded(tfull0 + 8 * acc, (it >> 1) & 1, abort_flag, p.err, p.timeout_ns);
        // the four warps of a group go on or leave together: they share barriers
        ok = group_agrees(1 + group, __shfl_sync(0xffffffffu, got, 0) != 0);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int u = 0; u < C::TURNS; ++u) {
          if (group + C::GROUPS * u >= chunks) continue;
          const uint32_t from = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * C::COLS + (group + C::GROUPS * u) * 32;
#pragma unroll
          for (int b = 0; b < 32; b += 8) {
            uint32_t v[C::PARTS][8];
#pragma unroll
            for (int part = 0; part < C::PARTS; ++part) tmem_ld8(from + part * p.n + b, v[part]);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              float x = __uint_as_float(v[0][j]);
              if (F32) x += __uint_as_float(v[1 % C::PARTS][j]) + __uint_as_float(v[2 % C::PARTS][j]);
              run[u][b + j] = first ? run[u][b + j] + x : x;
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty0 + 8 * acc);
      }
      if (!ok) break;
#pragma unroll
      for (int u = 0; u < C::TURNS; ++u) {
        const int chunk = group + C::GROUPS * u;
        if (GRAD && chunk == C::GROUPS - 1 && rows_zero > C::GROUPS * 32) g_vector(p, out, c0 + 32 * q, c1, C::GROUPS * 32 + r, false);
        if (chunk >= chunks) {
          if (GRAD && chunk * 32 < rows_zero) g_vector(p, out, c0 + 32 * q, c1, chunk * 32 + r, false);
          continue;
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) out[j * kHfOutLd + t] = run[u][j];
        named_bar_sync(1 + group, 128);
        const int m = chunk * 32 + r;
        const float* row = out + r * kHfOutLd;
        if (GRAD) {
          g_vector(p, row + 32 * q, c0 + 32 * q, c1, m, m < count);
          named_bar_sync(1 + group, 128);
          continue;
        }
        float f[32], now = top[u];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          f[i] = c0 + 4 * i + q < c1 ? row[4 * i + q] : -INFINITY;
          now = fmaxf(now, f[i]);
        }
        // NaN logits leave the maximum but reach the sum; a maximum of -inf subtracts nothing
        if (now > top[u]) {
          sum[u] *= top[u] == -INFINITY ? 0.f : ex2_approx((top[u] - now) * c);
          top[u] = now;
        }
        const float base = now == -INFINITY ? 0.f : now;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i & 3] += ex2_approx((f[i] - base) * c);
        sum[u] += (s[0] + s[1]) + (s[2] + s[3]);
        if (q == 0 && m < count) {
          const int64_t line = (int64_t)p.rows[m] * p.k;
          for (; next[u] < p.k; ++next[u]) {
            const int cl = p.cls[line + next[u]];
            if (cl >= c1) break;
            p.picked[line + next[u]] = row[cl - c0];
          }
        }
        named_bar_sync(1 + group, 128);
      }
    }
#pragma unroll
    for (int u = 0; u < (GRAD ? 0 : C::TURNS); ++u) {
      const int m = (group + C::GROUPS * u) * 32 + r;
      float most = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 1));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
      float s = sum[u] * (top[u] == most ? 1.f : ex2_approx((top[u] - most) * c));
      s += __shfl_xor_sync(0xffffffffu, s, 1);
      s += __shfl_xor_sync(0xffffffffu, s, 2);
      if (q == 0 && m < count) p.rec[(int64_t)blockIdx.x * p.cap + m] = make_float2(most, s);
    }
  } else if (F32) {
    // ------------------------------------------------------------ the head's parts
    const int w = warp - 2 - C::EPI, k4 = lane & 15, r0 = w * 16 + (lane >> 4);
    int stage = 0;
    uint32_t phase = 0;
    const int total = tiles * nkb;
    float4 f[8];
    int c0 = c_begin, k0 = 0;   // of the block that is loaded next
    const int last = GRAD ? min(c_end, p.V) : c_end;
    auto load = [&](float4 (&g)[8]) {
      const int k = k0 + 4 * k4;
      const float* src = p.w + (int64_t)(c0 + r0) * p.d + k;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        g[j] = c0 + r0 + 2 * j < last && k < p.d ? *reinterpret_cast<const float4*>(src + (int64_t)(2 * j) * p.d) : make_float4(0.f, 0.f, 0.f, 0.f);
      k0 += kHfK;
      if (k0 >= p.d) {
        k0 = 0;
        c0 += kHfM;
      }
    };
    auto put = [&](const float4 (&g)[8]) {
      int got = 0;
      if (lane == 0) got = mbar_wait_bounded(empty0 + 8 * stage, phase ^ 1, abort_flag, p.err, p.timeout_ns);
      if (!__shfl_sync(0xffffffffu, got, 0)) return false;
      uint8_t* at = smem + stage * stage_bytes;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = r0 + 2 * j;
        float x[4] = {g[j].x, g[j].y, g[j].z, g[j].w};
        uint8_t* to = at + row * 128 + (((k4 >> 1) ^ (row & 7)) << 4) + (k4 & 1) * 8;
#pragma unroll
        for (int q = 0; q < 3; ++q) {
          uint2 u;
          u.x = next_parts(x[0], x[1]);
          u.y = next_parts(x[2], x[3]);
          *reinterpret_cast<uint2*>(to + q * kHfPart) = u;
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(full0 + 8 * stage);
      if (++stage == stages) { stage = 0; phase ^= 1; }
      return true;
    };
    load(f);
    for (int i = 0; i < total && put(f); ++i) load(f);
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 2 * C::COLS);
  }
}

// G of the n_g classes from v_g (0: a forward pass over all).
template <bool F32, bool GRAD>
cudaError_t launch_few(const Head& a, int64_t v_g, int n_g, const Dev& dev, int* records) {
  const cudaError_t e = allow_smem<head_few_kernel<F32, GRAD>, HfCfg<F32>::SMEM>();
  if (e != cudaSuccess) return e;
  HfDev p = {};
  p.n = (int)((a.n + 15) / 16 * 16);
  p.n_rows = (int)a.n;
  CUtensorMap th, ta = {}, tw = {}, tw1 = {};
  if (!make_tmap_bf16(&th, a.packed, (uint64_t)a.cap * (F32 ? 3 : 1), (uint64_t)a.ld, (uint64_t)a.ld, kHfK, (uint32_t)p.n))
    return cudaErrorInvalidValue;
  if (!F32 && (!make_tmap_bf16(&ta, a.h, (uint64_t)a.n, (uint64_t)a.d, (uint64_t)a.d, kHfK, (uint32_t)p.n) ||
               !make_tmap_bf16(&tw, a.w, (uint64_t)a.V, (uint64_t)a.d, (uint64_t)a.d, kHfK, kHfM) ||
               !make_tmap_bf16(&tw1, a.w, (uint64_t)a.V, (uint64_t)a.d, (uint64_t)a.d, kHfK, kHfUnit)))
    return cudaErrorInvalidValue;
  p.count = a.count;
  p.rows = a.rows;
  p.w = static_cast<const float*>(a.w);
  p.cap = a.cap;
  p.d = a.d;
  p.V = a.V;
  p.inv_t = 1.f / a.temp;
  p.cls = a.cls;
  p.k = a.k;
  p.rec = a.rec;
  p.picked = a.picked;
  p.err = dev.err;
  p.timeout_ns = kWaitTimeoutNs;
  p.v0 = (int)v_g;
  p.v1 = GRAD ? (int)(v_g + (n_g + 63) / 64 * 64) : a.V;   // the products of G take 64 classes at a time
  p.pw = a.p;
  p.lse = a.lse;
  p.g = a.g;
  p.g_ref = a.g_ref;
  p.G = static_cast<bf16*>(a.G[0]);
  p.ld_g = a.piece;
  *records = (int)std::min<int64_t>(std::min(dev.num_sms, kHeadFewCtas), ((int64_t)(p.v1 - p.v0) + kHfUnit - 1) / kHfUnit);
  return launch_pdl(head_few_kernel<F32, GRAD>, dim3((unsigned)*records), dim3(HfCfg<F32>::THREADS), HfCfg<F32>::SMEM, dev.stream, th, ta, tw, tw1, p);
}

}  // namespace

cudaError_t head_few(int dtype, const Head& a, const Dev& dev, int* records) {
  return dtype == kBF16 ? launch_few<false, false>(a, 0, 0, dev, records) : launch_few<true, false>(a, 0, 0, dev, records);
}

cudaError_t head_few_grad(const Head& a, int64_t v_g, int n_g, const Dev& dev) {
  int ctas;
  return launch_few<true, true>(a, v_g, n_g, dev, &ctas);
}

}  // namespace adadsf
