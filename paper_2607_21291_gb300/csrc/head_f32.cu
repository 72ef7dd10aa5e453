// Products of the losses at the LM head for fp32 storage, on CUDA cores: the tiles of head_tc.cu
// (stats, G, dH, dW), 128 x 128 a block of 256 threads, 8 x 8 sums a thread in packed multiply-adds.
//
// A stage holds 16 k of both operands as [k][128 rows or columns] in shared memory, two stages; a
// thread loads the next one into registers while it works on the present one. An operand whose rows run
// along k (rows x features for logits, G for dH) is turned on its way into shared memory, the others
// are copied as they lie. A warp's 32 lanes are 2 x 16 of the tile's threads, so a k costs it six
// wavefronts of shared memory for 64 cycles of multiply-adds. One tile a block, dealt out by the hardware.
#include <algorithm>

#include "head.cuh"

namespace adadsf {
namespace {

constexpr int kHfTile = 128, kHfK = 16, kHfLd = kHfTile + 4;
enum { kStats = 0, kG = 1, kDH = 2, kDW = 3 };

struct HfDev {
  const float *h, *w;        // packed rows, head
  const float* Gd;           // the piece of dH and dW
  const int32_t *count, *rows;
  int64_t cap;
  int d, V;
  float inv_t, temp;
  const int32_t* cls;
  const float* p;
  int k;
  float2* rec;
  float* picked;
  const float *lse, *g;
  int v_g, n_g, v_d, n_d;    // first class and classes of the G piece, of the dH and dW piece (0: none)
  int splits, want_h, want_w, first, add_w, piece;
  float *G, *acc, *dw;
};

// One operand of a tile: 128 rows of it along m from m0 (rows from `ms` on read as zero), k up to ke.
struct Operand {
  const float* base;
  int64_t ld;
  int m0, ms, ke;
  bool along_k;              // a row is one m
};

__device__ __forceinline__ void load_stage(const Operand& o, int k0, int tid, float4 (&f)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = tid + i * 256;
    int m, k;
    if (o.along_k) {
      m = o.m0 + (j >> 2);
      k = k0 + (j & 3) * 4;
    } else {
      m = o.m0 + (j & 31) * 4;
      k = k0 + (j >> 5);
    }
    const bool in = m < o.ms && k < o.ke;
    f[i] = in ? *reinterpret_cast<const float4*>(o.base + (o.along_k ? m * o.ld + k : k * o.ld + m)) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
}
__device__ __forceinline__ void store_stage(const Operand& o, int tid, const float4 (&f)[2], float* s) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = tid + i * 256;
    if (o.along_k) {
      float* at = s + (j & 3) * 4 * kHfLd + (j >> 2);
      at[0] = f[i].x;
      at[kHfLd] = f[i].y;
      at[2 * kHfLd] = f[i].z;
      at[3 * kHfLd] = f[i].w;
    } else {
      *reinterpret_cast<float4*>(s + (j >> 5) * kHfLd + (j & 31) * 4) = f[i];
    }
  }
}

template <bool GRAD>
__global__ void __launch_bounds__(256, 2) head_f32_kernel(const __grid_constant__ HfDev p) {
  __shared__ __align__(16) float sa[2][kHfK * kHfLd], sb[2][kHfK * kHfLd];
  pdl_wait();
  pdl_trigger();
  const int count = *p.count, tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int mbs = (count + kHfTile - 1) / kHfTile;
  const int nbd = (p.d + kHfTile - 1) / kHfTile;
  const int vt_d = GRAD ? (p.n_d + kHfTile - 1) / kHfTile : 0;
  const int vt_g = ((GRAD ? p.n_g : p.V) + kHfTile - 1) / kHfTile;
  const int n_h = GRAD && p.want_h && p.n_d > 0 ? mbs * nbd * p.splits : 0, n_w = GRAD && p.want_w ? vt_d * nbd : 0;
  int t = blockIdx.x;
  if (t >= n_h + n_w + mbs * vt_g) return;
  int kind, m0, n0, slot = 0, k0 = 0, k1;
  Operand a, b;
  if (t < n_h) {
    kind = kDH;
    m0 = t % mbs * kHfTile;
    const int r = t / mbs;
    slot = r / nbd;
    n0 = (r - slot * nbd) * kHfTile;
    const int kbs = (p.n_d + kHfK - 1) / kHfK;
    k0 = (int)((int64_t)kbs * slot / p.splits) * kHfK;
    k1 = min(p.n_d, (int)((int64_t)kbs * (slot + 1) / p.splits) * kHfK);
    // G's columns past the last class up to a multiple of 4 are zero; the head has no such rows
    a = {p.Gd, p.piece, m0, count, k1, true};
    b = {p.w + (int64_t)p.v_d * p.d, p.d, n0, p.d, k1, false};
  } else if (t - n_h < n_w) {
    t -= n_h;
    kind = kDW;
    const int r = t / nbd;
    n0 = (t - r * nbd) * kHfTile;
    m0 = r * kHfTile;
    k1 = count;
    a = {p.Gd, p.piece, m0, p.piece, k1, false};
    b = {p.h, p.d, n0, p.d, k1, false};
  } else {
    t -= n_h + n_w;
    kind = GRAD ? kG : kStats;
    m0 = t % mbs * kHfTile;
    n0 = t / mbs * kHfTile;
    k1 = p.d;
    const int v0 = GRAD ? p.v_g : 0;
    a = {p.h, p.d, m0, count, k1, true};
    b = {p.w + (int64_t)v0 * p.d, p.d, n0, p.V - v0, k1, true};
  }
  float2 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = make_float2(0.f, 0.f);
  float4 fa[2], fb[2];
  if (k0 < k1) {
    load_stage(a, k0, tid, fa);
    load_stage(b, k0, tid, fb);
    store_stage(a, tid, fa, sa[0]);
    store_stage(b, tid, fb, sb[0]);
  }
  __syncthreads();
  int buf = 0;
  for (int k = k0; k < k1; k += kHfK) {
    const bool more = k + kHfK < k1;
    if (more) {
      load_stage(a, k + kHfK, tid, fa);
      load_stage(b, k + kHfK, tid, fb);
    }
#pragma unroll
    for (int kk = 0; kk < kHfK; ++kk) {
      float va[8], vb[8];
      load4(sa[buf] + kk * kHfLd + ty * 4, va);
      load4(sa[buf] + kk * kHfLd + 64 + ty * 4, va + 4);
      load4(sb[buf] + kk * kHfLd + tx * 4, vb);
      load4(sb[buf] + kk * kHfLd + 64 + tx * 4, vb + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 ai = make_float2(va[i], va[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __ffma2_rn(ai, make_float2(vb[2 * j], vb[2 * j + 1]), acc[i][j]);
      }
    }
    if (more) {
      store_stage(a, tid, fa, sa[buf ^ 1]);
      store_stage(b, tid, fb, sb[buf ^ 1]);
    }
    __syncthreads();
    buf ^= 1;
  }
  // sums of row m0 + (i & 4) * 16 + ty * 4 + (i & 3), columns n0 + {0, 64} + tx * 4 + {0 .. 3}
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int m = m0 + (i & 4) * 16 + ty * 4 + (i & 3);
    float f[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[2 * j] = acc[i][j].x;
      f[2 * j + 1] = acc[i][j].y;
    }
    if (kind == kDH || kind == kDW) {
      if (kind == kDH ? m >= count : p.v_d + m >= p.V) continue;
      float* row = kind == kDH ? p.acc + ((int64_t)slot * p.cap + m) * p.d : p.dw + (int64_t)(p.v_d + m) * p.d;
      const bool add = kind == kDH ? !p.first : p.add_w != 0;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int n = n0 + q * 64 + tx * 4;
        if (n >= p.d) continue;
        if (add) {
          float old[4];
          load4(row + n, old);
#pragma unroll
          for (int l = 0; l < 4; ++l) f[4 * q + l] += old[l];
        }
        *reinterpret_cast<float4*>(row + n) = make_float4(f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]);
      }
      continue;
    }
    const bool live = m < count;
    const int64_t row = live ? p.rows[m] : 0;
    const int32_t* cls = p.cls + row * p.k;
    const int c0 = (GRAD ? p.v_g : 0) + n0;
    int j = live ? first_class(cls, p.k, c0) : p.k;
    if (!GRAD) {
      float top = -INFINITY;
#pragma unroll
      for (int l = 0; l < 8; ++l) {
        if (c0 + (l >> 2) * 64 + tx * 4 + (l & 3) >= p.V) f[l] = -INFINITY;
        top = fmaxf(top, f[l]);
      }
      for (; j < p.k && cls[j] < c0 + kHfTile && cls[j] < p.V; ++j) {
        const int in = cls[j] - c0;
        if (((in & 63) >> 2) != tx) continue;
#pragma unroll
        for (int l = 0; l < 8; ++l)
          if (in == (l >> 2) * 64 + tx * 4 + (l & 3)) p.picked[row * p.k + j] = f[l];
      }
      top = max16(top);
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
#pragma unroll
      for (int l = 0; l < 8; ++l) sum += expf((f[l] - base) * p.inv_t);
      sum = sum16(sum);
      if (live && tx == 0) p.rec[(int64_t)(n0 / kHfTile) * p.cap + m] = make_float2(top, sum);
    } else {
      if (!live) continue;
      const float lse = p.lse[row], g = (p.g ? p.g[row] : 1.f) * p.temp;
#pragma unroll
      for (int l = 0; l < 8; ++l)
        f[l] = c0 + (l >> 2) * 64 + tx * 4 + (l & 3) < p.V ? expf(fmaf(f[l], p.inv_t, -lse)) : 0.f;
      for (; j < p.k && cls[j] < c0 + kHfTile && cls[j] < p.V; ++j) {
        const int in = cls[j] - c0;
        if (((in & 63) >> 2) != tx) continue;
        const float want = p.p ? p.p[row * p.k + j] : 1.f;
#pragma unroll
        for (int l = 0; l < 8; ++l)
          if (in == (l >> 2) * 64 + tx * 4 + (l & 3)) f[l] -= want;
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float4 v = make_float4(f[4 * q] * g, f[4 * q + 1] * g, f[4 * q + 2] * g, f[4 * q + 3] * g);
        const int n = n0 + q * 64 + tx * 4;
        if (p.v_g + n + 3 >= p.V) {   // no class: zero, whatever g is
          if (p.v_g + n >= p.V) v.x = 0.f;
          if (p.v_g + n + 1 >= p.V) v.y = 0.f;
          if (p.v_g + n + 2 >= p.V) v.z = 0.f;
          v.w = 0.f;
          if (p.v_g + n + 3 < p.V) v.w = f[4 * q + 3] * g;
        }
        *reinterpret_cast<float4*>(p.G + (int64_t)m * p.piece + n) = v;
      }
    }
  }
}

HfDev head_dev(const Head& a) {
  HfDev p = {};
  p.h = static_cast<const float*>(a.packed);
  p.w = static_cast<const float*>(a.w);
  p.count = a.count;
  p.rows = a.rows;
  p.cap = a.cap;
  p.d = a.d;
  p.V = a.V;
  p.inv_t = 1.f / a.temp;
  p.temp = a.temp;
  p.cls = a.cls;
  p.p = a.p;
  p.k = a.k;
  p.rec = a.rec;
  p.picked = a.picked;
  p.lse = a.lse;
  p.g = a.g;
  p.piece = a.piece;
  return p;
}

int64_t ceil_div64(int64_t a, int b) { return (a + b - 1) / b; }

}  // namespace

cudaError_t head_f32_stats(const Head& a, const Dev& dev) {
  const int64_t tiles = ceil_div64(a.n, kHfTile) * ceil_div64(a.V, kHfTile);
  if (tiles > INT32_MAX) return cudaErrorInvalidValue;
  return launch_pdl(head_f32_kernel<false>, dim3((unsigned)tiles), dim3(256), 0, dev.stream, head_dev(a));
}

cudaError_t head_f32_grad(const Head& a, int buf, int64_t v_g, int n_g, int64_t v_d, int n_d, bool first, const Dev& dev) {
  HfDev p = head_dev(a);
  p.Gd = static_cast<const float*>(a.G[buf ^ 1]);
  p.G = static_cast<float*>(a.G[buf]);
  p.v_g = (int)v_g;
  p.n_g = n_g;
  p.v_d = (int)v_d;
  p.n_d = n_d;
  p.splits = a.splits;
  p.want_h = a.dh != nullptr;
  p.want_w = a.dw != nullptr;
  p.first = first;
  p.add_w = a.add_w;
  p.acc = a.dh_acc;
  p.dw = static_cast<float*>(a.dw);
  const int64_t mbs = ceil_div64(a.n, kHfTile), nbd = ceil_div64(a.d, kHfTile);
  const int64_t tiles = mbs * ceil_div64(n_g, kHfTile) + (p.want_h && n_d ? mbs * nbd * a.splits : 0) +
                        (p.want_w ? ceil_div64(n_d, kHfTile) * nbd : 0);
  if (tiles == 0) return cudaSuccess;
  if (tiles > INT32_MAX) return cudaErrorInvalidValue;
  return launch_pdl(head_f32_kernel<true>, dim3((unsigned)tiles), dim3(256), 0, dev.stream, p);
}

}  // namespace adadsf
