// LayerNorm and RMSNorm of rows with the statistics that a backward pass needs, and that pass.
//   xhat = (x - mean) rstd, y = xhat w + b;   a = dy w
//   dx = rstd (a - mean(a) - xhat mean(a xhat)) + add,  dw = sum dy xhat,  db = sum dy  over the rows
// (RMSNorm: mean = 0, no b, no mean(a).) Both are bound by memory: each tensor is read once and written once.
//
// A group of threads takes a row, a thread the same columns of every row of its group, so that the
// weights and the sums of their gradients stay in its registers; sums of a row go over its warps
// through shared memory. The next rows' values are on their way while a row is worked on. Every group
// leaves its weight gradients, which a second kernel adds in order: results are the same in every run.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "internal.h"

namespace adadsf {
namespace {

constexpr int kNgThreads = 512;   // at most, of a block

struct NgDev {
  const void *x, *w, *b, *dy, *add;
  int64_t n;
  int d, group, groups;           // threads a group, groups a block
  float eps;
  float *mean, *rstd;             // mean null: RMSNorm
  void *y, *dx;
  float *pw, *pb;                 // [groups of all blocks][d]; null: not wanted
};


// Sums of S values over a group, in a fixed order; every thread gets them. `slot` alternates, so that one
// barrier a sum is enough.
template <int S>
__device__ __forceinline__ void group_sum(float (&v)[S], float* red, int slot, int group, int g, int warp_in_group, int lane) {
#pragma unroll
  for (int s = 0; s < S; ++s) v[s] = warp_sum(v[s]);
  if (group == 32) return;
  const int warps = group >> 5;
  float* r = red + ((slot & 1) * 16 + g * warps) * S;   // at most 16 warps a block
  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < S; ++s) r[warp_in_group * S + s] = v[s];
  }
  named_bar_sync(1 + g, group);
#pragma unroll
  for (int s = 0; s < S; ++s) v[s] = 0.f;
  for (int i = 0; i < warps; ++i) {
#pragma unroll
    for (int s = 0; s < S; ++s) v[s] += r[i * S + s];
  }
}

template <typename T, int NV>
__global__ void __launch_bounds__(kNgThreads) norm_forward_kernel(const __grid_constant__ NgDev p) {
  constexpr int V = Elem<T>::kVec;
  __shared__ float red[2 * 16];
  pdl_wait();
  pdl_trigger();
  const int g = threadIdx.x / p.group, t = threadIdx.x - g * p.group, lane = threadIdx.x & 31, wig = t >> 5;
  const int nv = p.d / V;
  const int64_t step = (int64_t)gridDim.x * p.groups;
  const float inv_d = 1.f / (float)p.d;
  uint4 wv[NV], bv[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.group;
    wv[i] = c < nv ? static_cast<const uint4*>(p.w)[c] : make_uint4(0, 0, 0, 0);
    bv[i] = c < nv && p.b ? static_cast<const uint4*>(p.b)[c] : make_uint4(0, 0, 0, 0);
  }
  uint4 next[NV];
  auto load = [&](int64_t r) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * p.group;
      next[i] = r < p.n && c < nv ? static_cast<const uint4*>(p.x)[r * nv + c] : make_uint4(0, 0, 0, 0);
    }
  };
  int64_t row = (int64_t)blockIdx.x * p.groups + g;
  load(row);
  int slot = 0;
  for (; row < p.n; row += step) {
    float x[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) unpack16(next[i], x[i], T());
    load(row + step);
    float mean = 0.f;
    if (p.mean) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) s[0] += x[i][j];
      group_sum<1>(s, red, slot++, p.group, g, wig, lane);
      mean = s[0] * inv_d;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in = t + i * p.group < nv;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        x[i][j] -= mean;
        if (in) q[0] = fmaf(x[i][j], x[i][j], q[0]);
      }
    }
    group_sum<1>(q, red, slot++, p.group, g, wig, lane);
    const float rstd = 1.f / sqrtf(q[0] * inv_d + p.eps);
    if (t == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * p.group;
      float w[V], b[V], y[V];
      unpack16(wv[i], w, T());
      unpack16(bv[i], b, T());
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = fmaf(x[i][j] * rstd, w[j], b[j]);
      if (c < nv) static_cast<uint4*>(p.y)[row * nv + c] = pack16(y, T());
    }
  }
}

template <typename T, int NV, bool ADD>
__global__ void __launch_bounds__(kNgThreads) norm_backward_kernel(const __grid_constant__ NgDev p) {
  constexpr int V = Elem<T>::kVec;
  __shared__ float red[2 * 16 * 2];
  pdl_wait();
  pdl_trigger();
  const int g = threadIdx.x / p.group, t = threadIdx.x - g * p.group, lane = threadIdx.x & 31, wig = t >> 5;
  const int nv = p.d / V;
  const int64_t step = (int64_t)gridDim.x * p.groups;
  const float inv_d = 1.f / (float)p.d;
  uint4 wv[NV];
  float sw[NV][V], sb[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.group;
    wv[i] = c < nv ? static_cast<const uint4*>(p.w)[c] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < V; ++j) sw[i][j] = sb[i][j] = 0.f;
  }
  uint4 nx[NV], ny[NV], na[NV];
  float n_mean = 0.f, n_rstd = 0.f;
  auto load = [&](int64_t r) {
    const bool row_in = r < p.n;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * p.group;
      const bool in = row_in && c < nv;
      nx[i] = in ? static_cast<const uint4*>(p.x)[r * nv + c] : make_uint4(0, 0, 0, 0);
      ny[i] = in ? static_cast<const uint4*>(p.dy)[r * nv + c] : make_uint4(0, 0, 0, 0);
      if (ADD) na[i] = in ? static_cast<const uint4*>(p.add)[r * nv + c] : make_uint4(0, 0, 0, 0);
    }
    n_mean = row_in && p.mean ? p.mean[r] : 0.f;
    n_rstd = row_in ? p.rstd[r] : 0.f;
  };
  int64_t row = (int64_t)blockIdx.x * p.groups + g;
  constexpr bool AHEAD = NV <= 2;   // wider rows have no registers for the next one
  if (AHEAD) load(row);
  int slot = 0;
  for (; row < p.n; row += step) {
    if (!AHEAD) load(row);
    uint4 x[NV], y[NV], a[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = nx[i];
      y[i] = ny[i];
      if (ADD) a[i] = na[i];
    }
    const float mean = n_mean, rstd = n_rstd;
    if (AHEAD) load(row + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in = t + i * p.group < nv;
      float xf[V], yf[V], w[V];
      unpack16(x[i], xf, T());
      unpack16(y[i], yf, T());
      unpack16(wv[i], w, T());
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xh = in ? (xf[j] - mean) * rstd : 0.f, ag = yf[j] * w[j];
        s[0] += ag;
        s[1] = fmaf(ag, xh, s[1]);
        sw[i][j] = fmaf(yf[j], xh, sw[i][j]);
        sb[i][j] += yf[j];
      }
    }
    group_sum<2>(s, red, slot++, p.group, g, wig, lane);
    const float c1 = p.mean ? s[0] * inv_d : 0.f, c2 = s[1] * inv_d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * p.group;
      float xf[V], yf[V], w[V], o[V];
      unpack16(x[i], xf, T());
      unpack16(y[i], yf, T());
      unpack16(wv[i], w, T());
      if (ADD) unpack16(a[i], o, T());
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xh = (xf[j] - mean) * rstd;
        const float dx = rstd * (yf[j] * w[j] - c1 - xh * c2);
        o[j] = ADD ? dx + o[j] : dx;
      }
      if (c < nv) static_cast<uint4*>(p.dx)[row * nv + c] = pack16(o, T());
    }
  }
  const int64_t part = ((int64_t)blockIdx.x * p.groups + g) * p.d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * p.group;
    if (c >= nv) continue;
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      if (p.pw) *reinterpret_cast<float4*>(p.pw + part + c * V + j) = make_float4(sw[i][j], sw[i][j + 1], sw[i][j + 2], sw[i][j + 3]);
      if (p.pb) *reinterpret_cast<float4*>(p.pb + part + c * V + j) = make_float4(sb[i][j], sb[i][j + 1], sb[i][j + 2], sb[i][j + 3]);
    }
  }
}

// Sums of the groups' weight gradients: 32 columns a block, 32 slices of the groups, added in order.
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
constexpr int kNgMaxBlocks = 2 * 152;

NgPlan plan(int dtype, int64_t n, int d) {
  const int vecs = d / (dtype == kBF16 ? 8 : 4);
  NgPlan q;
  q.nv = 1;
  while (q.nv < 4 && (vecs + q.nv - 1) / q.nv > kNgThreads) q.nv *= 2;
  q.group = ((vecs + q.nv - 1) / q.nv + 31) / 32 * 32;
  q.groups = std::max(1, std::min(kNgThreads / q.group, 15));
  if (q.group == 32) q.groups = 16;
  // few rows: a block a row, so that more SMs share them
  while (q.groups > 1 && (n + q.groups - 1) / q.groups < 152) q.groups /= 2;
  q.blocks = (int)std::max<int64_t>(1, std::min<int64_t>((n + q.groups - 1) / q.groups, kNgMaxBlocks));
  return q;
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
  // a block has at most 16 groups, the last one some without a row
  return (size_t)std::min<int64_t>(n + 15, (int64_t)kNgMaxBlocks * 16) * d * 2 * sizeof(float);
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
    return launch_pdl(norm_forward_kernel<decltype(t), decltype(nv)::value>, dim3(q.blocks), dim3(q.group * q.groups), 0,
                      dev.stream, p);
  });
}

cudaError_t norm_backward(int dtype, const void* dy, const void* x, const void* w, const float* mean, const float* rstd,
                          const void* add, int64_t n, int d, void* dx, float* dw, float* db, bool accumulate, float* scratch,
                          const Dev& dev) {
  const NgPlan q = plan(dtype, n, d);
  const int parts = q.blocks * q.groups;
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
  cudaError_t e = by_form(dtype, q.nv, [&](auto t, auto nv) {
    using T = decltype(t);
    constexpr int NV = decltype(nv)::value;
    const dim3 grid(q.blocks), block(q.group * q.groups);
    return add ? launch_pdl(norm_backward_kernel<T, NV, true>, grid, block, 0, dev.stream, p)
               : launch_pdl(norm_backward_kernel<T, NV, false>, grid, block, 0, dev.stream, p);
  });
  if (e != cudaSuccess || (!dw && !db)) return e;
  return launch_pdl(norm_weight_kernel, dim3((unsigned)((d + 31) / 32), 2), dim3(1024), 0, dev.stream, (const float*)p.pw,
                    (const float*)p.pb, parts, d, dw, db, accumulate ? 1 : 0);
}

}  // namespace adadsf
