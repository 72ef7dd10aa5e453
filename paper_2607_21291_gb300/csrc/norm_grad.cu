// LayerNorm and RMSNorm of rows with the statistics that a backward pass needs, and that pass.
//   xhat = (x - mean) rstd, y = xhat w + b;   a = dy w
//   dx = rstd (a - mean(a) - xhat mean(a xhat)) + add,  dw = sum dy xhat,  db = sum dy  over the rows
// (RMSNorm: mean = 0, no b, no mean(a).) Both are bound by memory: each tensor is read once and written once.
//
// A group of threads takes a row, a thread the same columns of every row of its group, so that the
// weights and the sums of their gradients stay in its registers; sums of a row go over its warps
// through shared memory. A thread copies what it will read of the next rows into a ring of its own
// (asynchronous copies, ng_depth rows in all: nobody else reads it, so no barrier guards it), which keeps enough
// bytes on their way whatever the registers allow. Every block leaves its weight gradients,
// which a second kernel adds in order: results are the same in every run.
// 65536 x 3584 bf16 with a sum: RMSNorm 160 us forward, 308 backward (5.9 and 6.1 TB/s); LayerNorm 190 and 328, whose forward pass has two
// sums one after the other; 24 x 768 11 us for both, two launches.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "internal.h"

namespace adadsf {
namespace {

// Threads of a block, at most. Of one vector a thread two blocks share an SM, with 72 registers a thread: with 64 the
// next rows' statistics were spilled, which waits for them (388 -> 711 us at 65536 x 3584). LayerNorm's gradient of bf16 rows takes
// one row at a time for the same reason (two: 484 us, one: 328).
constexpr int ng_threads(int nv) { return nv == 1 ? 448 : 512; }
constexpr int kNgOneLaunch = 32;   // blocks up to which the last one adds the weights' gradients
constexpr int ng_rows(int nv) { return nv <= 2 ? 2 : 1; }   // a group works on at a time: their sums share a barrier
// Rows of a thread's ring, for N tensors of NV vectors: what two blocks an SM (NV 1) have room for.
constexpr int ng_depth(int n, int nv) { return n == 1 ? (nv <= 2 ? 8 / nv : 4) : nv <= 2 ? 4 : 2; }

struct NgDev {
  const void *x, *w, *b, *dy, *add;
  int64_t n;
  int d, group, groups;           // threads a group, groups a block
  float eps;
  float *mean, *rstd;             // mean null: RMSNorm
  void *y, *dx;
  float *pw, *pb;                 // [blocks][d]; null: not wanted
  float *dw, *db;
  int accumulate;
  int* arrived;                   // the block that comes last adds the blocks' parts; null: norm_weight_kernel does
};


// 16 bytes as pairs of floats, and back: arithmetic in packed pairs, since a row's instructions, not
// its bytes, would bound the backward pass (568 -> 467 us at 65536 x 3584 with the forward pass).
template <int P>
__device__ __forceinline__ void pairs(const uint4& u, float2 (&f)[P]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < P; ++i)
    f[i] = P == 4 ? make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u))
                  : make_float2(__uint_as_float(w[2 * (i & 1)]), __uint_as_float(w[2 * (i & 1) + 1]));
}
template <int P>
__device__ __forceinline__ uint4 unpairs(const float2 (&f)[P]) {
  if (P == 4) return make_uint4(pack_bf16x2(f[0].x, f[0].y), pack_bf16x2(f[1].x, f[1].y), pack_bf16x2(f[2 % P].x, f[2 % P].y),
                                pack_bf16x2(f[3 % P].x, f[3 % P].y));
  return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// Sums of S (1, 2 or 4) values over a warp: lanes halve their values before they halve their distance, so that four sums
// take 6 shuffles in place of 20. The lane gets the sum of value lane * S / 32.
template <int S>
__device__ __forceinline__ float warp_sums(const float (&v)[S], int lane) {
  float k[S];
#pragma unroll
  for (int s = 0; s < S; ++s) k[s] = v[s];
  int distance = 16;
#pragma unroll
  for (int n = S; n > 1; n >>= 1, distance >>= 1) {
    const bool upper = lane & distance;
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
      const float send = upper ? k[i] : k[i + n / 2], keep = upper ? k[i + n / 2] : k[i];
      k[i] = keep + __shfl_xor_sync(0xffffffffu, send, distance);
    }
  }
#pragma unroll
  for (int o = 16 / S; o > 0; o >>= 1) k[0] += __shfl_xor_sync(0xffffffffu, k[0], o);
  return k[0];
}

// Sums of S values over a group, in a fixed order; every thread gets them. `turn` alternates, so that one
// barrier a sum is enough.
template <int S>
__device__ __forceinline__ void group_sum(float (&v)[S], float* red, int turn, int group, int g, int warp_in_group, int lane) {
  constexpr int LANES = 32 / S;   // of a value
  float mine = warp_sums(v, lane);
  const int warps = group >> 5, value = lane / LANES, w = lane % LANES;
  if (warps > 1) {
    float* r = red + ((turn & 1) * 16 + g * warps) * S;   // at most 16 warps a block
    if (w == 0) r[warp_in_group * S + value] = mine;
    named_bar_sync(1 + g, group);
    mine = w < warps ? r[w * S + value] : 0.f;
    if (LANES < 16 && w + LANES < warps) mine += r[(w + LANES) * S + value];
#pragma unroll
    for (int o = (LANES < 16 ? LANES : 16) / 2; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  }
#pragma unroll
  for (int s = 0; s < S; ++s) v[s] = __shfl_sync(0xffffffffu, mine, s * LANES);
}

// A thread's ring: N tensors' vectors of ng_depth rows, of which the ones ahead are on their way.
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid ? 4 : 0) : "memory");
}
__device__ __forceinline__ float ring_float(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
template <int N, int NV>
struct NgRing {
  uint32_t base;       // of this thread's first 16 bytes
  int threads;
  __device__ __forceinline__ uint32_t at(int slot, int tensor, int i) const {
    return base + 16u * (uint32_t)(((slot * N + tensor) * NV + i) * threads);
  }
  __device__ __forceinline__ uint4 read(int slot, int tensor, int i) const {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at(slot, tensor, i)) : "memory");
    return v;
  }
};

template <typename T, int NV>
__global__ void __launch_bounds__(ng_threads(NV), NV == 1 ? 2 : 1) norm_forward_kernel(const __grid_constant__ NgDev p) {
  constexpr int V = Elem<T>::kVec, DEPTH = ng_depth(1, NV), ROWS = ng_rows(NV);
  extern __shared__ __align__(16) uint8_t ring_smem[];
  __shared__ float red[2 * 16 * ROWS];
  pdl_wait();
  pdl_trigger();
  const int g = threadIdx.x / p.group, t = threadIdx.x - g * p.group, lane = threadIdx.x & 31, wig = t >> 5;
  const int nv = p.d / V;
  const int64_t step = (int64_t)gridDim.x * p.groups;
  const float inv_d = 1.f / (float)p.d;
  const NgRing<1, NV> ring = {smem_u32(ring_smem) + 16u * threadIdx.x, (int)blockDim.x};
  const uint4* x_all = static_cast<const uint4*>(p.x);
  auto fetch = [&](int64_t r, int slot) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * p.group;
      const bool in = r < p.n && c < nv;
      cp_async16(ring.at(slot, 0, i), x_all + (in ? r * nv + c : 0), in);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int64_t row = (int64_t)blockIdx.x * p.groups + g;
  constexpr int AHEAD = DEPTH - ROWS;
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) fetch(row + k * step, k);
  uint4 wv[NV], bv[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.group;
    wv[i] = c < nv ? static_cast<const uint4*>(p.w)[c] : make_uint4(0, 0, 0, 0);
    bv[i] = c < nv && p.b ? static_cast<const uint4*>(p.b)[c] : make_uint4(0, 0, 0, 0);
  }
  int slot = 0, turn = 0;
  for (; row < p.n; row += ROWS * step) {
#pragma unroll
    for (int k = 0; k < ROWS; ++k) fetch(row + (AHEAD + k) * step, (slot + AHEAD + k) % DEPTH);
    asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
    constexpr int P = V / 2;
    float2 x[ROWS][NV][P];
    float mean[ROWS] = {}, q[ROWS] = {};
#pragma unroll
    for (int k = 0; k < ROWS; ++k)
#pragma unroll
      for (int i = 0; i < NV; ++i) pairs(ring.read((slot + k) % DEPTH, 0, i), x[k][i]);
    slot = (slot + ROWS) % DEPTH;
    if (p.mean) {
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
        float2 m = both(0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < P; ++j) m = __fadd2_rn(m, x[k][i][j]);
        mean[k] = m.x + m.y;
      }
      group_sum<ROWS>(mean, red, turn++, p.group, g, wig, lane);
#pragma unroll
      for (int k = 0; k < ROWS; ++k) mean[k] *= inv_d;
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      float2 s = both(0.f);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool in = t + i * p.group < nv;
#pragma unroll
        for (int j = 0; j < P; ++j) {
          x[k][i][j] = in ? __fadd2_rn(x[k][i][j], both(-mean[k])) : both(0.f);
          s = __ffma2_rn(x[k][i][j], x[k][i][j], s);
        }
      }
      q[k] = s.x + s.y;
    }
    group_sum<ROWS>(q, red, turn++, p.group, g, wig, lane);
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int64_t r = row + k * step;
      if (r >= p.n) break;
      const float rstd = 1.f / sqrtf(q[k] * inv_d + p.eps);
      if (t == 0) {
        if (p.mean) p.mean[r] = mean[k];
        p.rstd[r] = rstd;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = t + i * p.group;
        float2 w[P], b[P], y[P];
        pairs(wv[i], w);
        pairs(bv[i], b);
#pragma unroll
        for (int j = 0; j < P; ++j) y[j] = __ffma2_rn(__fmul2_rn(x[k][i][j], both(rstd)), w[j], b[j]);
        if (c < nv) static_cast<uint4*>(p.y)[r * nv + c] = unpairs(y);
      }
    }
  }
}

template <typename T, int NV, bool ADD, bool MEAN>
__global__ void __launch_bounds__(ng_threads(NV), NV == 1 ? 2 : 1) norm_backward_kernel(const __grid_constant__ NgDev p) {
  constexpr int V = Elem<T>::kVec, N = ADD ? 3 : 2, DEPTH = ng_depth(N, NV), ROWS = MEAN && V == 8 ? 1 : ng_rows(NV);
  extern __shared__ __align__(16) uint8_t ring_smem[];
  __shared__ float red[2 * 16 * 2 * ROWS];
  pdl_wait();
  pdl_trigger();
  const int g = threadIdx.x / p.group, t = threadIdx.x - g * p.group, lane = threadIdx.x & 31, wig = t >> 5;
  const int nv = p.d / V;
  const int64_t step = (int64_t)gridDim.x * p.groups;
  const float inv_d = 1.f / (float)p.d;
  const NgRing<N, NV> ring = {smem_u32(ring_smem) + 16u * threadIdx.x, (int)blockDim.x};
  // the rows' statistics [slot][mean, rstd]: a copy a warp, RMSNorm's one number a copy a thread (302 against 325 us at
  // 65536 x 3584)
  const uint32_t stats = smem_u32(ring_smem) + 16u * DEPTH * N * NV * blockDim.x + 8u * DEPTH * (MEAN ? threadIdx.x >> 5 : threadIdx.x);
  const uint4 *x_all = static_cast<const uint4*>(p.x), *y_all = static_cast<const uint4*>(p.dy),
              *a_all = static_cast<const uint4*>(p.add);
  auto fetch = [&](int64_t r, int slot) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * p.group;
      const bool in = r < p.n && c < nv;
      const int64_t at = in ? r * nv + c : 0;
      cp_async16(ring.at(slot, 0, i), x_all + at, in);
      cp_async16(ring.at(slot, 1, i), y_all + at, in);
      if (ADD) cp_async16(ring.at(slot, N - 1, i), a_all + at, in);
    }
    const bool row_in = r < p.n;
    if (!MEAN || lane == 0) {
      if (MEAN) cp_async4(stats + 8u * slot, p.mean + (row_in ? r : 0), row_in);
      cp_async4(stats + 8u * slot + 4, p.rstd + (row_in ? r : 0), row_in);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int64_t row = (int64_t)blockIdx.x * p.groups + g;
  constexpr int AHEAD = DEPTH - ROWS;
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) fetch(row + k * step, k);
  constexpr int P = V / 2;
  uint4 wv[NV];
  float2 sw[NV][P], sb[MEAN ? NV : 1][P];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.group;
    wv[i] = c < nv ? static_cast<const uint4*>(p.w)[c] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < P; ++j) sw[i][j] = sb[MEAN ? i : 0][j] = both(0.f);
  }
  int slot = 0, turn = 0;
  for (; row < p.n; row += ROWS * step) {
#pragma unroll
    for (int k = 0; k < ROWS; ++k) fetch(row + (AHEAD + k) * step, (slot + AHEAD + k) % DEPTH);
    asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
    if (MEAN) __syncwarp();   // lane 0's copies of the statistics
    constexpr int S = MEAN ? 2 : 1;
    // fp32: xhat = (x - mean) rstd, the difference first as in the forward pass, since x rstd - mean rstd is off by roundings
    // of the mean's size (rows of a mean of 1000 and a spread of 2: the weights' gradient of one row 3e-5, now 1e-7). bf16: x rstd +
    // shift, an instruction less a pair (327 us in place of 347 at 65536 x 3584): of rows in 8 bits the mean is some 2^8
    // spreads at most as a rule, and the gradients of rows are rounded by 2^-8.
    constexpr bool APART = MEAN && V == 4;
    float shift[ROWS], rstd[ROWS], s[S * ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const uint32_t st = stats + 8u * ((slot + k) % DEPTH);
      rstd[k] = ring_float(st + 4);
      shift[k] = !MEAN ? 0.f : APART ? -ring_float(st) : -ring_float(st) * rstd[k];
      float2 sa = both(0.f), sx = both(0.f);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        // vectors past the row and rows past the last are zeros in dy: they add nothing
        float2 x[P], y[P], w[P];
        pairs(ring.read((slot + k) % DEPTH, 0, i), x);
        pairs(ring.read((slot + k) % DEPTH, 1, i), y);
        pairs(wv[i], w);
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const float2 xh = APART ? __fmul2_rn(__fadd2_rn(x[j], both(shift[k])), both(rstd[k]))
                            : MEAN ? __ffma2_rn(x[j], both(rstd[k]), both(shift[k])) : __fmul2_rn(x[j], both(rstd[k]));
          const float2 a = __fmul2_rn(y[j], w[j]);
          if (MEAN) sa = __fadd2_rn(sa, a);
          sx = __ffma2_rn(a, xh, sx);
          sw[i][j] = __ffma2_rn(y[j], xh, sw[i][j]);
          if (MEAN) sb[MEAN ? i : 0][j] = __fadd2_rn(sb[MEAN ? i : 0][j], y[j]);
        }
      }
      s[S * k] = sx.x + sx.y;
      if (MEAN) s[S * k + S - 1] = sa.x + sa.y;
    }
    group_sum<S * ROWS>(s, red, turn++, p.group, g, wig, lane);
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int64_t r = row + k * step;
      if (r < p.n) {
        // dx = rstd a + (x by + c1): by = -rstd^2 mean(a xhat), c1 = -rstd (shift mean(a xhat) + mean(a)); apart, x - mean for x
        // and no shift
        const float c2 = -(s[S * k] * inv_d) * rstd[k], by = c2 * rstd[k];
        const float c1 = MEAN ? fmaf(c2, APART ? 0.f : shift[k], -(s[S * k + S - 1] * inv_d) * rstd[k]) : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = t + i * p.group;
          float2 x[P], y[P], w[P], o[P];
          pairs(ring.read((slot + k) % DEPTH, 0, i), x);
          pairs(ring.read((slot + k) % DEPTH, 1, i), y);
          pairs(wv[i], w);
          if (ADD) pairs(ring.read((slot + k) % DEPTH, N - 1, i), o);
#pragma unroll
          for (int j = 0; j < P; ++j) {
            const float2 xm = APART ? __fadd2_rn(x[j], both(shift[k])) : x[j];
            const float2 rest = MEAN ? __ffma2_rn(xm, both(by), both(c1)) : __fmul2_rn(xm, both(by));
            const float2 dx = __ffma2_rn(__fmul2_rn(y[j], w[j]), both(rstd[k]), rest);
            o[j] = ADD ? __fadd2_rn(dx, o[j]) : dx;
          }
          if (c < nv) static_cast<uint4*>(p.dx)[r * nv + c] = unpairs(o);
        }
      }
    }
    slot = (slot + ROWS) % DEPTH;
  }
  if (!p.pw && !p.pb) return;
  // the block's groups, in order, through the ring's memory
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  float* part = reinterpret_cast<float*>(ring_smem);   // [group][NV][V][threads of a group]
#pragma unroll
  for (int which = 0; which < (MEAN ? 2 : 1); ++which) {
    float* dst = which ? p.pb : p.pw;
    if (!dst) continue;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float2& v = which ? sb[MEAN ? i : 0][j / 2] : sw[i][j / 2];
        part[((g * NV + i) * V + j) * p.group + t] = j & 1 ? v.y : v.x;
      }
    __syncthreads();
    if (g == 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = t + i * p.group;
        if (c >= nv) continue;
        float s[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          s[j] = 0.f;
          for (int q = 0; q < p.groups; ++q) s[j] += part[((q * NV + i) * V + j) * p.group + t];
        }
        float* at = dst + (int64_t)blockIdx.x * p.d + c * V;
#pragma unroll
        for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(at + j) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
      }
    }
  }
  if (!p.arrived) return;
  __shared__ int last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.arrived, 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  if (threadIdx.x == 0) *p.arrived = 0;   // as it was found
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float* src = which ? p.pb : p.pw;
    float* dst = which ? p.db : p.dw;
    if (!dst) continue;
    for (int c = 4 * threadIdx.x; c < p.d; c += 4 * blockDim.x) {
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      float old[4] = {};
      if (p.accumulate)
        for (int j = 0; j < 4; ++j) old[j] = dst[c + j];
#pragma unroll
      for (int i = 0; i < kNgOneLaunch; ++i) {
        const float4 f = i < (int)gridDim.x ? __ldcg(reinterpret_cast<const float4*>(src + (int64_t)i * p.d + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
        s.x += f.x;
        s.y += f.y;
        s.z += f.z;
        s.w += f.w;
      }
      const float sum[4] = {s.x, s.y, s.z, s.w};
      for (int j = 0; j < 4; ++j) dst[c + j] = old[j] + sum[j];   // grad_w may start at any float
    }
  }
}

// Sums of the blocks' weight gradients: 32 columns a block, 32 slices of the parts, added in order.
__global__ void __launch_bounds__(1024)
    norm_weight_kernel(const float* pw, const float* pb, int parts, int d, float* dw, float* db, int accumulate) {
  pdl_wait();
  pdl_trigger();
  __shared__ float red[32][33];
  const float* src = blockIdx.y ? pb : pw;
  float* dst = blockIdx.y ? db : dw;
  if (!dst) return;
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < d) {
#pragma unroll 4
    for (int i = slice; i < parts; i += 32) s += src[(int64_t)i * d + c];
  }
  red[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && c < d) {
    float sum = accumulate ? dst[c] : 0.f;
    for (int i = 0; i < 32; ++i) sum += red[i][lane];
    dst[c] = sum;
  }
}

struct NgPlan {
  int group, groups, nv, blocks;
};
constexpr int kNgMaxBlocks = 3 * 152;

NgPlan plan(int dtype, int64_t n, int d) {
  const int vecs = d / (dtype == kBF16 ? 8 : 4);
  NgPlan q;
  q.nv = 1;
  while (q.nv < 4 && (vecs + q.nv - 1) / q.nv > ng_threads(q.nv)) q.nv *= 2;
  q.group = ((vecs + q.nv - 1) / q.nv + 31) / 32 * 32;
  q.groups = ng_threads(q.nv) / q.group;
  // few rows: a block a row, so that more SMs share them
  while (q.groups > 1 && (n + q.groups - 1) / q.groups < 152) q.groups /= 2;
  // what an SM has registers for (72 a thread of one vector)
  const int per_sm = q.nv == 1 ? std::max(2, 896 / (q.group * q.groups)) : 1;
  q.blocks = (int)std::min<int64_t>((n + q.groups - 1) / q.groups, 152 * per_sm);
  return q;
}

// KERNEL with the rings of its threads: N tensors of NV vectors.
template <auto KERNEL, int N, int NV>
cudaError_t start(const NgPlan& q, const NgDev& p, const Dev& dev) {
  constexpr int kThread = ng_depth(N, NV) * (N * NV * 16 + (N > 1 ? 8 : 0));   // with the rows' statistics
  static_assert(N == 1 || kThread >= NV * 8 * 4, "a ring holds its thread's weight gradients");
  const cudaError_t e = allow_smem<KERNEL, ng_threads(NV) * kThread>();
  const int threads = q.group * q.groups;
  return e != cudaSuccess ? e : launch_pdl(KERNEL, dim3(q.blocks), dim3(threads), (size_t)threads * kThread, dev.stream, p);
}

// f(type, vectors a thread): kNormMaxD is 2 of 8 or 4 of 4 values for every thread of a block.
template <typename F>
cudaError_t by_form(int dtype, int nv, F f) {
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  if (dtype == kBF16) return nv == 1 ? f(bf16(), One()) : f(bf16(), Two());
  return nv == 1 ? f(0.f, One()) : nv == 2 ? f(0.f, Two()) : f(0.f, std::integral_constant<int, 4>());
}

}  // namespace

size_t norm_backward_scratch(int64_t n, int d) {
  return (size_t)std::min<int64_t>(n, kNgMaxBlocks) * d * 2 * sizeof(float);
}

cudaError_t norm_forward(int dtype, const void* x, const void* w, const void* b, int64_t n, int d, float eps, bool rms, void* y,
                         float* mean, float* rstd, const Dev& dev) {
  const NgPlan q = plan(dtype, n, d);
  NgDev p = {};
  p.x = x;
  p.w = w;
  p.b = b;
  p.n = n;
  p.d = d;
  p.group = q.group;
  p.groups = q.groups;
  p.eps = eps;
  p.mean = rms ? nullptr : mean;
  p.rstd = rstd;
  p.y = y;
  return by_form(dtype, q.nv, [&](auto t, auto nv) {
    return start<norm_forward_kernel<decltype(t), decltype(nv)::value>, 1, decltype(nv)::value>(q, p, dev);
  });
}

cudaError_t norm_backward(int dtype, const void* dy, const void* x, const void* w, const float* mean, const float* rstd,
                          const void* add, int64_t n, int d, void* dx, float* dw, float* db, bool accumulate, int* sync,
                          float* scratch, const Dev& dev) {
  const NgPlan q = plan(dtype, n, d);
  const int parts = q.blocks;
  NgDev p = {};
  p.x = x;
  p.w = w;
  p.dy = dy;
  p.add = add;
  p.n = n;
  p.d = d;
  p.group = q.group;
  p.groups = q.groups;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.dx = dx;
  p.pw = dw ? scratch : nullptr;
  p.pb = db ? scratch + (int64_t)parts * d : nullptr;
  p.dw = dw;
  p.db = db;
  p.accumulate = accumulate;
  const bool one_launch = parts <= kNgOneLaunch;
  p.arrived = one_launch ? sync : nullptr;
  cudaError_t e = by_form(dtype, q.nv, [&](auto t, auto nv) {
    using T = decltype(t);
    constexpr int NV = decltype(nv)::value;
    if (mean) return add ? start<norm_backward_kernel<T, NV, true, true>, 3, NV>(q, p, dev)
                         : start<norm_backward_kernel<T, NV, false, true>, 2, NV>(q, p, dev);
    return add ? start<norm_backward_kernel<T, NV, true, false>, 3, NV>(q, p, dev)
               : start<norm_backward_kernel<T, NV, false, false>, 2, NV>(q, p, dev);
  });
  if (e != cudaSuccess || one_launch || (!dw && !db)) return e;
  return launch_pdl(norm_weight_kernel, dim3((unsigned)((d + 31) / 32), 2), dim3(1024), 0, dev.stream, (const float*)p.pw,
                    (const float*)p.pb, parts, d, dw, db, accumulate ? 1 : 0);
}

}  // namespace adadsf
