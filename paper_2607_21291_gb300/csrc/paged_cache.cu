// Paged cache: rotary, quantisation and write of new tokens, and the read back.
//
// A block takes up to kPgRows packed rows; its first warp finds where they lie, a lane a row. A thread holds
// sixteen features of a head's vector in two chunks whose features pair in the rotation (or neighbours), and
// a warp four or eight heads of a row at a time, head after head, so a row's turns stay in registers. Products and sums
// of the rotation are separate fp32 ones. 8-bit storage: the largest |x| of the vector by
// shuffles on the bits of |x| (a NaN is larger than any number there), then round(x * (127 (1 / m))).
// Bytes bound both kernels: each element is read and written once. 8192 new rows of the Qwen2.5-7B shape into
// 8 bits take 30 us (4.8 TB/s), 32768 read back 18.5 us (5.5 TB/s); stored as bf16 29 us (5.2) and 24 us (5.6). The Pythia-70M
// shape (fp32): 19 and 46 us (5.3, 5.8), in 8 bits 14 and 46 us (5.3, 3.7). One row a block, with the turns read again for
// each chunk, took 58 and (eight features a thread, four rows a block) 40 us.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace adadsf {
namespace {

constexpr int kPgThreads = 256;
constexpr int kPgRows = 16;   // most rows of a block
// Resident blocks an SM, as the registers of this way of loading (a thread's features, turns and results) allow: fewer
// leave loads out of flight, more make the compiler spill.
constexpr int kPgAppendPerSm = 4, kPgReadPerSm = 8;
constexpr float kPgTiny = 7.888609052210118e-31f;   // 2^-100: vectors below are stored as zeros

// Eight features e0 .. e0 + 7 of `src`.
template <typename T>
__device__ __forceinline__ void load8(const T* src, float* f) {
#pragma unroll
  for (int i = 0; i < 8; i += Elem<T>::kVec) unpack16(__ldg(reinterpret_cast<const uint4*>(src + i)), f + i, T());
}
template <typename T>
__device__ __forceinline__ void store8(T* dst, const float* f) {
#pragma unroll
  for (int i = 0; i < 8; i += Elem<T>::kVec) store_vec(dst + i, f + i);
}

// Features e0 .. e0 + 7 of a head turned one by one (half not a multiple of 8): (a c - b s, b c + a s) for the
// pair (a, b), each product and sum rounded by itself.
template <typename T>
__device__ __forceinline__ void turned8(const T* head, int e0, int half, const float2* tab, float* f) {
  load8(head + e0, f);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = e0 + i;
    if (e >= 2 * half) break;
    const bool lower = e < half;
    const float g = Elem<T>::to_f(head[lower ? e + half : e - half]);
    const float2 cs = tab[lower ? e : e - half];
    const float t = __fmul_rn(g, cs.y);
    f[i] = __fadd_rn(__fmul_rn(f[i], cs.x), lower ? -t : t);
  }
}

// Where a block's rows lie: number of the token's vector of head 0 (-1: no token, or a page that is not),
// and its place. Whole first warp; then for all. Meanwhile the other warps of the grid's first block look at the
// counts of all sequences: the rows only lead to those that have some.
struct PgRows {
  int64_t vec[kPgRows];
  int place[kPgRows];
};
__device__ __forceinline__ void pg_rows(const Paged& p, int64_t row0, int n, PgRows& s, int* err) {
  const int lane = threadIdx.x;
  if (lane < 32) {
    int b = paged_find(p, row0, lane);
    if (lane < n) {
      const int64_t row = row0 + lane;
      while (b < p.B && p.starts[b + 1] <= row) ++b;
      int place = -1, page = -1;
      if (b < p.B) {
        const PagedSeq q = paged_seq(p, b, err);
        const int i = (int)(row - q.row0);
        if (i >= 0 && i < q.n) place = q.len - q.n + i;
        if (place >= 0) page = paged_page(p, b, place, err);
      }
      s.vec[lane] = page >= 0 ? paged_vec(p, page, place, 0) : -1;
      s.place[lane] = place;
    }
  } else if (blockIdx.x == 0 && blockIdx.y == 0) {
    for (int b = threadIdx.x - 32; b < p.B; b += kPgThreads - 32) paged_seq(p, b, err);
  }
  __syncthreads();
}

template <typename T, int HD, bool I8>
__global__ void __launch_bounds__(kPgThreads, kPgAppendPerSm)
    paged_append_kernel(const Paged p, const T* qkv, const float2* tab, int half, int n_pos, const int32_t* pos,
                        T* q_out, int rows, int* err) {
  constexpr int TPV = HD / 16;          // threads of a vector, two chunks of eight features each
  constexpr int VPW = 32 / TPV;         // vectors of a warp at a time: a group of a row's heads
  __shared__ PgRows s;
  __shared__ int at_s[kPgRows];
  pdl_wait();
  pdl_trigger();
  const int64_t row0 = (int64_t)blockIdx.x * rows;
  const int n = (int)min((int64_t)rows, p.n_rows - row0);
  const int tid = threadIdx.x, lane = tid & 31, j = lane % TPV;
  if (half > 0 && pos && tid >= 32 && tid < 32 + n) at_s[tid - 32] = pos[row0 + tid - 32];
  pg_rows(p, row0, n, s, err);
  const int heads = p.Hq + 2 * p.Hkv, first = q_out ? 0 : p.Hq, groups = (heads - first + VPW - 1) / VPW;
  const bool even = (half & 7) == 0;
  // chunks whose features pair: j and j + half / 8; behind the rotated ones, neighbours
  const int pairs = even ? half / 8 : 0;
  const bool turns = j < pairs;
  const int e0 = 8 * (turns ? j : 2 * j), e1 = 8 * (turns ? j + pairs : 2 * j + 1);
  // this warp's share of the units (row, group of heads): neighbours, so that a row's turns are read once
  const int total = n * groups, warps = gridDim.y * (kPgThreads / 32), me = blockIdx.y * (kPgThreads / 32) + tid / 32;
  const int u1 = (int)((int64_t)total * (me + 1) / warps);
  int row_in = -1, at = 0;
  float c[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = sn[i] = 0.f;
#pragma unroll 1
  for (int u = (int)((int64_t)total * me / warps); u < u1; ++u) {
    const int r = u / groups, h = first + (u - r * groups) * VPW + lane / TPV;
    const bool live = h < heads;
    const T* src = qkv + ((row0 + r) * heads + (live ? h : 0)) * HD;
    if (r != row_in && half > 0) {
      row_in = r;
      at = pos ? at_s[r] : max(s.place[r], 0);
      if (at < 0 || at >= n_pos) {
        set_device_error(err, DEVERR_INDEX);
        at = min(max(at, 0), n_pos - 1);
      }
      if (turns) {
        const float4* t4 = reinterpret_cast<const float4*>(tab + (int64_t)at * half + 8 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 x = __ldg(t4 + i);
          c[2 * i] = x.x;
          sn[2 * i] = x.y;
          c[2 * i + 1] = x.z;
          sn[2 * i + 1] = x.w;
        }
      }
    }
    float f[2][8];
    const bool rotated = h < p.Hq + p.Hkv && half > 0;
    if (rotated && !even) {
      turned8(src, e0, half, tab + (int64_t)at * half, f[0]);
      turned8(src, e1, half, tab + (int64_t)at * half, f[1]);
    } else {
      load8(src + e0, f[0]);
      load8(src + e1, f[1]);
      if (rotated && turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = f[0][i], y = f[1][i];
          f[0][i] = __fsub_rn(__fmul_rn(x, c[i]), __fmul_rn(y, sn[i]));
          f[1][i] = __fadd_rn(__fmul_rn(y, c[i]), __fmul_rn(x, sn[i]));
        }
      }
    }
    if (live && h < p.Hq) {
      T* dst = q_out + ((row0 + r) * p.Hq + h) * HD;
      store8(dst + e0, f[0]);
      store8(dst + e1, f[1]);
    }
    const bool cached = live && h >= p.Hq && s.vec[r] >= 0;
    const bool value = h >= p.Hq + p.Hkv;
    const int64_t vec = s.vec[r] + ((int64_t)(h - p.Hq - (value ? p.Hkv : 0)) << p.page_log2);
    if (!I8) {
      if (cached) {
        T* dst = static_cast<T*>(value ? p.v : p.k) + vec * HD;
        store8(dst + e0, f[0]);
        store8(dst + e1, f[1]);
      }
    } else if (__any_sync(0xffffffffu, cached)) {
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        m = max(m, max(__float_as_uint(f[0][i]) & 0x7fffffffu, __float_as_uint(f[1][i]) & 0x7fffffffu));
#pragma unroll
      for (int o = 1; o < TPV; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      if (cached) {
        const float most = __uint_as_float(m);
        const bool bad = m >= 0x7f800000u, none = most < kPgTiny;
        const float scale = bad ? NAN : none ? 0.f : __fdiv_rn(most, 127.f);
        const float inv = bad || none ? 0.f : __fmul_rn(__frcp_rn(most), 127.f);   // a reciprocal for the products, not a division
        uint32_t w[4] = {0, 0, 0, 0};
        if (!bad && !none) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            w[i >> 2] |= (uint32_t)(__float2int_rn(__fmul_rn(f[i >> 3][i & 7], inv)) & 0xff) << (8 * (i & 3));
        }
        int8_t* dst = static_cast<int8_t*>(value ? p.v : p.k) + vec * HD;
        *reinterpret_cast<uint2*>(dst + e0) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2*>(dst + e1) = make_uint2(w[2], w[3]);
        if (j == 0) (value ? p.vs : p.ks)[vec] = scale;
      }
    }
  }
}

template <typename T, int HD, bool I8>
__global__ void __launch_bounds__(kPgThreads, kPgReadPerSm)
    paged_read_kernel(const Paged p, T* k_out, T* v_out, int rows, int* err) {
  constexpr int FPT = I8 ? 16 : 8;   // features of a thread
  constexpr int TPV = HD / FPT;
  __shared__ PgRows s;
  pdl_wait();
  pdl_trigger();
  const int64_t row0 = (int64_t)blockIdx.x * rows;
  const int n = (int)min((int64_t)rows, p.n_rows - row0);
  pg_rows(p, row0, n, s, err);
  const int tid = threadIdx.x, e0 = tid % TPV * FPT, total = n * 2 * p.Hkv;
#pragma unroll 2
  for (int v = blockIdx.y * (kPgThreads / TPV) + tid / TPV; v < total; v += gridDim.y * (kPgThreads / TPV)) {
    const int r = v / (2 * p.Hkv), h = v - r * 2 * p.Hkv;
    const bool value = h >= p.Hkv;
    const int g = h - (value ? p.Hkv : 0);
    const int64_t at = s.vec[r], vec = at + ((int64_t)g << p.page_log2);
    T* dst = (value ? v_out : k_out) + ((row0 + r) * p.Hkv + g) * HD + e0;
    if (I8) {
      uint4 w = make_uint4(0, 0, 0, 0);
      float scale = 0.f;
      if (at >= 0) {
        w = __ldg(reinterpret_cast<const uint4*>(static_cast<const int8_t*>(value ? p.v : p.k) + vec * HD + e0));
        scale = __ldg((value ? p.vs : p.ks) + vec);
      }
      const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)(int8_t)(in[2 * k + (i >> 2)] >> (8 * (i & 3))) * scale;
        store8(dst + 8 * k, f);
      }
    } else {
      constexpr int N = 8 / Elem<T>::kVec;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const T*>(value ? p.v : p.k) + vec * HD + e0) + i;
        reinterpret_cast<uint4*>(dst)[i] = at >= 0 ? __ldg(src) : make_uint4(0, 0, 0, 0);
      }
    }
  }
}

// f(type, head size, storage) for the call's.
template <typename F>
cudaError_t with_kind(int dtype, const Paged& p, F&& f) {
  auto hd = [&](auto t, auto i8) -> cudaError_t {
    if (p.hd == 128) return f(t, std::integral_constant<int, 128>(), i8);
    if (p.hd == 64) return f(t, std::integral_constant<int, 64>(), i8);
    return cudaErrorInvalidValue;
  };
  if (dtype == kBF16) return p.i8 ? hd(bf16(), std::true_type()) : hd(bf16(), std::false_type());
  return p.i8 ? hd(0.f, std::true_type()) : hd(0.f, std::false_type());
}

}  // namespace

// Rows of a block (equal shares of as many full waves of `per_sm` blocks an SM as are needed), and where there
// are few rows, several blocks for the vectors of one.
static dim3 pg_grid(int64_t n_rows, int vectors, int per_pass, int per_sm, int num_sms, int* rows) {
  const int64_t wave = (int64_t)per_sm * num_sms, waves = (n_rows + kPgRows * wave - 1) / (kPgRows * wave);
  *rows = (int)((n_rows + waves * wave - 1) / (waves * wave));
  const int64_t blocks = (n_rows + *rows - 1) / *rows;
  const int64_t passes = ((int64_t)*rows * vectors + per_pass - 1) / per_pass;
  return dim3((unsigned)blocks, (unsigned)std::min<int64_t>(passes, std::max<int64_t>(1, wave / blocks)));
}

cudaError_t paged_append(int dtype, const Paged& p, const void* qkv, const float2* tab, int half, int n_pos,
                         const int32_t* pos, void* q_out, const Dev& dev) {
  return with_kind(dtype, p, [&](auto t, auto hd, auto i8) -> cudaError_t {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    int rows;
    const dim3 grid = pg_grid(p.n_rows, (q_out ? p.Hq : 0) + 2 * p.Hkv, kPgThreads / (HD / 16), kPgAppendPerSm, dev.num_sms, &rows);
    return launch_pdl(paged_append_kernel<T, HD, decltype(i8)::value>, grid, dim3(kPgThreads), 0, dev.stream, p,
                      static_cast<const T*>(qkv), tab, half, n_pos, pos, static_cast<T*>(q_out), rows, dev.err);
  });
}

cudaError_t paged_read(int dtype, const Paged& p, void* k_out, void* v_out, const Dev& dev) {
  return with_kind(dtype, p, [&](auto t, auto hd, auto i8) -> cudaError_t {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    constexpr bool I8 = decltype(i8)::value;
    int rows;
    const dim3 grid = pg_grid(p.n_rows, 2 * p.Hkv, kPgThreads / (HD / (I8 ? 16 : 8)), kPgReadPerSm, dev.num_sms, &rows);
    return launch_pdl(paged_read_kernel<T, HD, I8>, grid, dim3(kPgThreads), 0, dev.stream, p, static_cast<T*>(k_out),
                      static_cast<T*>(v_out), rows, dev.err);
  });
}

}  // namespace adadsf
