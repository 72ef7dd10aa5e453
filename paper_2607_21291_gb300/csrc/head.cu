// Losses at the LM head: targets, packing of the rows that have one, and what joins the
// products of head_tc.cu (formulas in head.cuh).
#include <math.h>

#include <algorithm>

#include "head.cuh"

namespace adadsf {
namespace {

constexpr int kTeacherThreads = 128;

// A block a row. p = softmax of the slots in use, sorted by class (each slot counts the ones before
// it: k^2 comparisons, no barriers between them). 2400 rows of 64 slots: 16 us in each pass.
__global__ void __launch_bounds__(kTeacherThreads)
    head_teacher_kernel(const int32_t* idx, const float* logit, int k, int V, float inv_t, int32_t* cls, float* p, float* ent,
                        int32_t* target, int* err) {
  pdl_wait();
  pdl_trigger();
  __shared__ int32_t c[kHeadMaxK];
  __shared__ float t[kHeadMaxK];
  __shared__ float red[2][kTeacherThreads / 32];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float top = -INFINITY;
  bool bad = false;
  for (int j = tid; j < k; j += kTeacherThreads) {
    const int32_t id = idx[row * k + j];
    const float z = logit[row * k + j] * inv_t;
    const bool in = id >= 0 && id < V && !(z == -INFINITY);
    bad |= id >= V;
    c[j] = in ? id : INT_MAX;
    t[j] = in ? z : -INFINITY;
    if (in) top = fmaxf(top, z);
  }
  if (bad) set_device_error(err, DEVERR_INDEX);
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) red[0][warp] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  float sum = 0.f;
  for (int j = tid; j < k; j += kTeacherThreads) {
    if (c[j] != INT_MAX) sum += expf(t[j] - top);
  }
  sum = warp_sum(sum);
  if (lane == 0) red[1][warp] = sum;
  __syncthreads();
  sum = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  const float log_sum = logf(sum), inv = 1.f / sum;
  float e = 0.f;
  for (int j = tid; j < k; j += kTeacherThreads) {
    const int32_t mine = c[j];
    const bool in = mine != INT_MAX;
    const float w = in ? expf(t[j] - top) * inv : 0.f;
    if (in && w != 0.f) e += w * ((t[j] - top) - log_sum);
    int rank = 0;
    for (int i = 0; i < k; ++i) rank += c[i] < mine || (c[i] == mine && i < j);
    cls[row * k + rank] = mine;
    p[row * k + rank] = w;
    if (rank == 0) target[row] = in ? mine : -1;
  }
  e = warp_sum(e);
  __syncthreads();
  if (lane == 0) red[0][warp] = e;
  __syncthreads();
  if (tid == 0) ent[row] = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
}

constexpr int kPackThreads = 256;

// Rows with a target, in order: their numbers, their count and a copy of their features (of bf16 rows that all have one none). Every block counts all
// targets by itself (no launch before it, no order between blocks). Rows without one get a loss, a
// logarithm and a gradient of zero; what they hold is read by nobody. Packed rows past the last one, up to a
// multiple of kHeadZeroPad, are zero: products over rows run that far.
//
// The copy is bf16 [cap][ld]; of fp32 features three parts (see next_parts), each such a matrix, ld features with zeros behind
// the d-th. Backward: the largest weight of a row's loss as well. Bound by the copy: some 46000 of 57270 bf16 rows of 3784 142 us (4.9 TB/s);
// 24 rows of 768 3.5 us, a launch's latency.
constexpr int kPutAhead = 8;   // loads of a lane on their way
__device__ __forceinline__ void put_row(const bf16* src, bf16* dst, int64_t, int d, int, int lane) {
  const int nv = d / 8;
  for (int v = lane; v < nv; v += 32 * kPutAhead) {
    uint4 u[kPutAhead];
#pragma unroll
    for (int j = 0; j < kPutAhead; ++j)
      if (v + 32 * j < nv) u[j] = reinterpret_cast<const uint4*>(src)[v + 32 * j];
#pragma unroll
    for (int j = 0; j < kPutAhead; ++j)
      if (v + 32 * j < nv) reinterpret_cast<uint4*>(dst)[v + 32 * j] = u[j];
  }
}
// 4 features of fp32 into the parts, `part` elements apart.
__device__ __forceinline__ void put4(const float4& f, bf16* dst, int64_t part) {
  float x[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    uint2 u;
    u.x = next_parts(x[0], x[1]);
    u.y = next_parts(x[2], x[3]);
    *reinterpret_cast<uint2*>(dst + q * part) = u;
  }
}
__device__ __forceinline__ void put_row(const float* src, bf16* dst, int64_t part, int d, int ld, int lane) {
  for (int v = lane; v < ld / 4; v += 32 * kPutAhead) {
    float4 f[kPutAhead];
#pragma unroll
    for (int j = 0; j < kPutAhead; ++j)
      f[j] = v + 32 * j < d / 4 ? reinterpret_cast<const float4*>(src)[v + 32 * j] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kPutAhead; ++j)
      if (v + 32 * j < ld / 4) put4(f[j], dst + 4 * (v + 32 * j), part);
  }
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads)
    head_pack_kernel(const int32_t* target, int64_t n, int V, int64_t per_block, const T* h, int d, bf16* packed, int64_t cap,
                     int ld, int32_t* rows, int32_t* count, const float* g, float* g_ref, float* loss, float* lse, T* dh, int* err) {
  pdl_wait();
  pdl_trigger();
  constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
  constexpr int W = kPackThreads / 32;
  __shared__ int red[2][W];
  __shared__ int at[kPackThreads];
  __shared__ float most[W];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t r0 = blockIdx.x * per_block, r1 = min(n, r0 + per_block);
  int before = 0, all = 0;
  float top = 0.f;
  const bool weigh = g && blockIdx.x == 0;
#pragma unroll 8
  for (int64_t i = tid; i < n; i += kPackThreads) {
    const int32_t t = target[i];
    const int in = t >= 0 && t < V;
    all += in;
    before += in && i < r0;
    if (weigh && in) top = fmaxf(top, fabsf(g[i]));
  }
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  before = __reduce_add_sync(0xffffffffu, before);
  all = __reduce_add_sync(0xffffffffu, all);
  if (lane == 0) {
    red[0][warp] = before;
    red[1][warp] = all;
    most[warp] = top;
  }
  __syncthreads();
  before = all = 0;
  for (int i = 0; i < W; ++i) {
    before += red[0][i];
    all += red[1][i];
  }
  if (blockIdx.x == 0 && tid == 0) {
    *count = all;
    if (g_ref) {
      for (int i = 0; i < W; ++i) top = fmaxf(top, most[i]);
      *g_ref = top > 0.f && top < INFINITY ? top : 1.f;
    }
  }
  const int nv = d / Elem<T>::kVec;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  for (int64_t c = r0; c < r1; c += kPackThreads) {
    const int64_t r = c + tid;
    const int32_t t = r < r1 ? target[r] : -1;
    const bool in = t >= 0 && t < V;
    if (t >= V) set_device_error(err, DEVERR_INDEX);
    const uint32_t live = __ballot_sync(0xffffffffu, in);
    __syncthreads();   // the counts and places before are read
    if (lane == 0) red[0][warp] = __popc(live);
    __syncthreads();
    int place = before + __popc(live & ((1u << lane) - 1));
    for (int i = 0; i < W; ++i) {
      if (i < warp) place += red[0][i];
      before += red[0][i];
    }
    at[tid] = in ? place : -1;
    if (in) rows[place] = (int32_t)r;
    if (r < r1 && !in) {
      if (loss) loss[r] = 0.f;
      if (lse) lse[r] = 0.f;
    }
    __syncthreads();
    const int in_chunk = (int)min((int64_t)kPackThreads, r1 - c);
    for (int i = warp; i < in_chunk; i += W) {
      if (PARTS == 1 && all == n) break;   // the products read the rows where they are
      if (at[i] >= 0) {
        put_row(h + (c + i) * d, packed + (int64_t)at[i] * ld, cap * ld, d, ld, lane);
      } else if (dh) {
        uint4* dst = reinterpret_cast<uint4*>(dh + (c + i) * d);
        for (int v = lane; v < nv; v += 32) dst[v] = zero;
      }
    }
  }
  if (PARTS == 1 && all == n) return;
  const int tail = (kHeadZeroPad - all % kHeadZeroPad) % kHeadZeroPad;
  for (int i = (int)(blockIdx.x + gridDim.x * warp); i < tail; i += (int)gridDim.x * W) {
    for (int q = 0; q < PARTS; ++q) {
      uint4* dst = reinterpret_cast<uint4*>(packed + (q * cap + all + i) * ld);
      for (int v = lane; v < ld / 8; v += 32) dst[v] = zero;
    }
  }
}

// The head's parts (fp32): [3][Vp][ld], zeros behind the d-th feature and the last class. 50304 x 512: 38 us for 258 MB read and
// written (6.8 TB/s).
__global__ void __launch_bounds__(256) head_split_kernel(const float* w, int V, int d, int Vp, int ld, bf16* parts) {
  pdl_wait();
  pdl_trigger();
  const int64_t n = (int64_t)Vp * (ld / 4), part = (int64_t)Vp * ld;
  const int nv = ld / 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / nv;
    const int c = (int)(i - r * nv) * 4;
    const bool in = r < V && c < d;
    put4(in ? *reinterpret_cast<const float4*>(w + r * d + c) : make_float4(0.f, 0.f, 0.f, 0.f), parts + r * ld + c, part);
  }
}

// Losses of 32 packed rows: a lane a row, the warps share the records of its classes and its targets.
// Every sum runs in one order. 4096 rows of 256 records: 8 us; 24 rows of 152: 6, latency.
constexpr int kMergeWarps = 32, kMergeAhead = 8;
__global__ void __launch_bounds__(32 * kMergeWarps)
    head_merge_kernel(const int32_t* count, const int32_t* rows, const float2* rec, int64_t cap, int n_rec, const float* picked,
                      const float* p, const float* ent, int k, float temp, float* loss, float* lse) {
  pdl_wait();
  pdl_trigger();
  __shared__ float s_top[kMergeWarps][32], s_sum[kMergeWarps][32], s_pz[kMergeWarps][32], s_p[kMergeWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = *count;
  const float inv_t = 1.f / temp, c = inv_t * 1.4426950408889634f;
  for (int64_t m0 = (int64_t)blockIdx.x * 32; m0 < n; m0 += (int64_t)gridDim.x * 32) {
    const int64_t m = m0 + lane;
    float top = -INFINITY, sum = 0.f, pz = 0.f, ps = 0.f;
    int64_t row = 0;
    if (m < n) {
      row = rows[m];
      for (int i = warp; i < n_rec; i += kMergeWarps * kMergeAhead) {
        float2 r[kMergeAhead];
        float now = top;
#pragma unroll
        for (int j = 0; j < kMergeAhead; ++j) {
          const int at = i + j * kMergeWarps;
          r[j] = at < n_rec ? rec[(int64_t)at * cap + m] : make_float2(-INFINITY, 0.f);
        }
#pragma unroll
        for (int j = 0; j < kMergeAhead; ++j) now = fmaxf(now, r[j].x);
        // a side without a number so far (-inf) adds nothing but its NaN
        sum *= top == now ? 1.f : ex2_approx((top - now) * c);
#pragma unroll
        for (int j = 0; j < kMergeAhead; ++j) sum += r[j].y * (r[j].x == now ? 1.f : ex2_approx((r[j].x - now) * c));
        top = now;
      }
      for (int j = warp; j < k; j += kMergeWarps) {
        const float w = p ? p[row * k + j] : 1.f;
        if (w != 0.f) {
          pz += w * (picked[row * k + j] * inv_t);
          ps += w;
        }
      }
    }
    s_top[warp][lane] = top;
    s_sum[warp][lane] = sum;
    s_pz[warp][lane] = pz;
    s_p[warp][lane] = ps;
    __syncthreads();
    if (warp == 0 && m < n) {
      for (int i = 1; i < kMergeWarps; ++i) top = fmaxf(top, s_top[i][lane]);
      sum = 0.f;
      pz = 0.f;
      ps = 0.f;
      for (int i = 0; i < kMergeWarps; ++i) {
        const float a = s_top[i][lane] == top ? 1.f : ex2_approx((s_top[i][lane] - top) * c);
        sum += s_sum[i][lane] * a;
        pz += s_pz[i][lane];
        ps += s_p[i][lane];
      }
      const float most = top * inv_t, rest = logf(sum);
      lse[row] = most + rest;
      // targets against the largest logit first: a target that is the largest leaves the sum's logarithm alone
      if (loss) loss[row] = temp * temp * ((ent ? ent[row] : 0.f) + ((ps * most - pz) + ps * rest));
    }
    __syncthreads();
  }
}

// acc[0] += sum of the losses, acc[1] += rows that have one; one block, in a fixed order.
__global__ void __launch_bounds__(1024) head_sum_kernel(const float* loss, int64_t n, const int32_t* count, double* acc) {
  pdl_wait();
  pdl_trigger();
  __shared__ double red[32];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += (double)loss[i];
  s = warp_sum(s);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 32; ++i) s += red[i];
    acc[0] += s;
    acc[1] += (double)*count;
  }
}

// The hidden states' gradient: a packed row's partial sums added in order, rounded once, to its row. 4096 rows of 3584 features in 4
// parts: 47 us for 264 MB (5.6 TB/s).
template <typename T>
__global__ void __launch_bounds__(256)
    head_finish_kernel(const float* acc, const int32_t* count, const int32_t* rows, int64_t cap, int d, int splits,
                       const float* g_ref, float temp, T* dh) {
  pdl_wait();
  pdl_trigger();
  const float scale = *g_ref * temp;
  constexpr int V = Elem<T>::kVec;
  const int nv = d / V;
  const int64_t n = (int64_t)*count * nv, stride = cap * d;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / nv;
    const int c = (int)(i - m * nv) * V;
    float s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
#pragma unroll 8
    for (int q = 0; q < splits; ++q) {
      const float* a = acc + q * stride + m * d + c;
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        float f[4];
        load4(a + j, f);
#pragma unroll
        for (int l = 0; l < 4; ++l) s[j + l] += f[l];
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] *= scale;
    store_vec(dh + (int64_t)rows[m] * d + c, s);
  }
}

template <typename T>
cudaError_t pack(const Head& a, bool backward, bool split, const Dev& dev) {
  const int64_t per = std::max<int64_t>(8, (a.n + 511) / 512);
  cudaError_t e = launch_pdl(head_pack_kernel<T>, dim3((unsigned)((a.n + per - 1) / per)), dim3(kPackThreads), 0, dev.stream,
                             a.target, a.n, a.V, per, static_cast<const T*>(a.h), a.d, static_cast<bf16*>(a.packed), a.cap, a.ld,
                             a.rows, a.count, backward ? a.g : (const float*)nullptr, backward ? a.g_ref : (float*)nullptr,
                             backward ? (float*)nullptr : a.loss, backward ? (float*)nullptr : a.lse,
                             backward ? static_cast<T*>(a.dh) : (T*)nullptr, dev.err);
  if (e != cudaSuccess || !split || sizeof(T) == 2) return e;
  const int64_t pieces = (int64_t)a.Vp * (a.ld / 4);
  return launch_pdl(head_split_kernel, dim3((unsigned)std::min<int64_t>((pieces + 255) / 256, 8 * dev.num_sms)), dim3(256), 0,
                    dev.stream, static_cast<const float*>(a.w), a.V, a.d, a.Vp, a.ld, static_cast<bf16*>(a.w_parts));
}

}  // namespace

// Classes a piece: 256 MB of G, 2048 at least (past 65536 bf16 rows more than that). With 96 MB the launches' first and last waves cost more than its second reading from the
// L2 saves (3 x 259 fp32 tokens 725 -> 650 us, 8 x 511 of the Pythia-1.4B head 1750 -> 1590); 600 and 1500 MB are no faster.
HeadPlan head_plan(int dtype, int64_t n, int d, int V) {
  const int64_t parts = dtype == kBF16 ? 1 : 3, tile = 256;
  HeadPlan q;
  q.cap = (n + kHeadRowPad - 1) / kHeadRowPad * kHeadRowPad;
  q.ld = (d + 7) / 8 * 8;
  q.Vp = (int)(((int64_t)V + 63) / 64 * 64);
  const int64_t padded = ((int64_t)V + 255) / 256 * 256;
  int64_t piece = std::max<int64_t>(2048, (256ll << 20) / std::max<int64_t>(1, q.cap * 2 * parts));
  const int64_t pieces = (padded + piece - 1) / piece;
  piece = ((padded + pieces - 1) / pieces + 255) / 256 * 256;
  q.piece = (int)piece;
  q.pieces = (int)((V + piece - 1) / piece);
  // dH sums over a piece's classes: cut so that its tiles are about as long as the others, into no more than four, or what
  // gives every pair of SMs two tiles where there are few rows (their parts are added up again)
  const int64_t other = std::max<int64_t>(std::max<int64_t>(q.cap, d), 1024);
  const int64_t tiles = std::max<int64_t>(1, q.cap / tile * ((d + tile - 1) / tile));
  int64_t splits = std::max<int64_t>(1, (piece + other / 2) / other);
  q.splits = (int)std::min<int64_t>(splits, std::max<int64_t>(4, (160 + tiles - 1) / tiles));
  q.packed = (size_t)(parts * q.cap * q.ld * 2);
  q.w_parts = dtype == kBF16 ? 0 : (size_t)(parts * q.Vp * q.ld * 2);
  q.rec = (size_t)(std::max<int64_t>(padded / 128, kHeadFewCtas) * q.cap * 8);
  q.g = (size_t)(parts * q.cap * piece * 2);
  q.acc = (size_t)(q.splits * q.cap * d * 4);
  return q;
}

cudaError_t head_teacher(const int32_t* idx, const float* logit, int64_t n, int k, int V, float temp, int32_t* cls, float* p,
                         float* ent, int32_t* target, const Dev& dev) {
  return launch_pdl(head_teacher_kernel, dim3((unsigned)n), dim3(kTeacherThreads), 0, dev.stream, idx, logit, k, V, 1.f / temp,
                    cls, p, ent, target, dev.err);
}

cudaError_t head_forward(int dtype, const Head& a, const Dev& dev) {
  const bool few = a.n <= (dtype == kBF16 ? kHeadFewRows : kHeadFewRowsF32);
  int records = (a.V + 127) / 128;
  cudaError_t e = dtype == kBF16 ? pack<bf16>(a, false, !few, dev) : pack<float>(a, false, !few, dev);
  if (e == cudaSuccess) e = few ? head_few(dtype, a, dev, &records) : head_stats(dtype, a, dev);
  if (e != cudaSuccess) return e;
  const int blocks = (int)std::min<int64_t>((a.n + 31) / 32, 2 * dev.num_sms);
  e = launch_pdl(head_merge_kernel, dim3((unsigned)blocks), dim3(32 * kMergeWarps), 0, dev.stream, (const int32_t*)a.count,
                 (const int32_t*)a.rows, (const float2*)a.rec, a.cap, records, (const float*)a.picked, a.p, a.ent, a.k,
                 a.temp, a.loss, a.lse);
  if (e != cudaSuccess || !a.acc) return e;
  return launch_pdl(head_sum_kernel, dim3(1), dim3(1024), 0, dev.stream, (const float*)a.loss, a.n, (const int32_t*)a.count, a.acc);
}

cudaError_t head_backward(int dtype, const Head& a, const HeadPlan& plan, const Dev& dev) {
  // The gradient's logits of few fp32 rows come from the kernel of their forward pass: at a target of nearly all the weight q - 1
  // is a difference of logits of both passes, and those of the other kernel, added up in another order, leave their
  // roundings (20 rows of 256 features, 5000 classes: head gradient 3.0e-6 off, so 1.4e-6). It is quicker as well: loss and
  // gradients of 77 rows at a 50304 x 512 head 285 -> 267 us. bf16 logits are one product a step, which both kernels add up in
  // the same chunks and order: the same bits.
  const bool few = dtype != kBF16 && a.n <= kHeadFewRowsF32;
  cudaError_t e = dtype == kBF16 ? pack<bf16>(a, true, true, dev) : pack<float>(a, true, !few || a.dh, dev);
  for (int j = 0; few && j < plan.pieces && e == cudaSuccess; ++j) {
    const int64_t v = (int64_t)j * plan.piece;
    const int n_v = (int)std::min<int64_t>(plan.piece, a.V - v);
    e = head_few_grad(a, v, n_v, dev);
    if (e == cudaSuccess) e = head_grad(dtype, a, 1, 0, 0, v, n_v, j == 0, dev);
  }
  // launch j: G of piece j, gradients of piece j - 1
  for (int j = 0; !few && j <= plan.pieces && e == cudaSuccess; ++j) {
    const int64_t v = (int64_t)j * plan.piece, before = v - plan.piece;
    const int n_g = j < plan.pieces ? (int)std::min<int64_t>(plan.piece, a.V - v) : 0;
    const int n_d = j > 0 ? (int)std::min<int64_t>(plan.piece, a.V - before) : 0;
    e = head_grad(dtype, a, j & 1, v, n_g, before, n_d, j == 1, dev);
  }
  if (e != cudaSuccess || !a.dh || a.dh_whole) return e;
  const int blocks = (int)std::min<int64_t>((a.n * a.d / 4 + 255) / 256, 8 * dev.num_sms);
  if (dtype == kBF16)
    return launch_pdl(head_finish_kernel<bf16>, dim3((unsigned)blocks), dim3(256), 0, dev.stream, (const float*)a.dh_acc,
                      (const int32_t*)a.count, (const int32_t*)a.rows, a.cap, a.d, a.splits, (const float*)a.g_ref,
                      a.temp, static_cast<bf16*>(a.dh));
  return launch_pdl(head_finish_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, dev.stream, (const float*)a.dh_acc,
                    (const int32_t*)a.count, (const int32_t*)a.rows, a.cap, a.d, a.splits, (const float*)a.g_ref,
                    a.temp, static_cast<float*>(a.dh));
}

}  // namespace adadsf
