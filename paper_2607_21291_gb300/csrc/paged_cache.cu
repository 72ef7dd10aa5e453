// Paged cache: rotary, quantisation and write of new tokens, and the read back.
//
// A thread holds eight features of one head's vector; the hd / 8 threads of a vector
// are neighbours in a warp. Rotation turns feature i with i + half (both read,
// so that no thread waits for another) in separate fp32 products and sums. 8-bit storage:
// the largest |x| of the vector by shuffles on the bits of |x| (a NaN is larger
// than any number there), then round(x * (127 / m)).
// Bytes bound both kernels: each element is read and written once.
#include <math.h>

#include <type_traits>

#include "paged.cuh"

namespace adadsf {
namespace {

constexpr int kPgThreads = 256;
constexpr float kPgTiny = 7.888609052210118e-31f;   // 2^-100: vectors below are stored as zeros

// Eight features e0 .. e0 + 7 of `src`.
template <typename T>
__device__ __forceinline__ void load8(const T* src, float* f) {
#pragma unroll
  for (int i = 0; i < 8; i += Elem<T>::kVec) load_vec(src + i, f + i);
}
template <typename T>
__device__ __forceinline__ void store8(T* dst, const float* f) {
#pragma unroll
  for (int i = 0; i < 8; i += Elem<T>::kVec) store_vec(dst + i, f + i);
}

// Features e0 .. e0 + 7 of a head, turned: (a c - b s, b c + a s) for the pair (a, b), each
// product and sum rounded by itself.
template <typename T>
__device__ __forceinline__ void turned8(const T* head, int e0, int half, const float2* tab, float* f) {
  load8(head + e0, f);
  if (e0 >= 2 * half) return;
  if ((half & 7) == 0) {
    const bool lower = e0 < half;
    float g[8];
    load8(head + (lower ? e0 + half : e0 - half), g);
    const float4* t4 = reinterpret_cast<const float4*>(tab + (lower ? e0 : e0 - half));
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float4 cs = t4[i / 2];
      const float t0 = __fmul_rn(g[i], cs.y), t1 = __fmul_rn(g[i + 1], cs.w);
      f[i] = __fadd_rn(__fmul_rn(f[i], cs.x), lower ? -t0 : t0);
      f[i + 1] = __fadd_rn(__fmul_rn(f[i + 1], cs.z), lower ? -t1 : t1);
    }
    return;
  }
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

template <typename T, int HD, bool I8>
__global__ void __launch_bounds__(kPgThreads)
    paged_append_kernel(const Paged p, const T* qkv, const float2* tab, int half, int n_pos, const int32_t* pos,
                        T* q_out, int* err) {
  constexpr int TPV = HD / 8;   // threads of a vector
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 31;
  const int heads = p.Hq + 2 * p.Hkv;
  // the row's sequence and place: every warp finds them for itself
  const int b = paged_find(p, row, lane);
  int place = -1, page = -1;
  if (b < p.B) {
    const PagedSeq s = paged_seq(p, b, err);
    const int i = (int)(row - s.row0);
    if (i >= 0 && i < s.n) place = s.len - s.n + i;
    if (place >= 0) page = paged_page(p, b, place, err);
  }
  const float2* turn = tab;
  if (half > 0) {
    int at = pos ? pos[row] : max(place, 0);
    if (at < 0 || at >= n_pos) {
      set_device_error(err, DEVERR_INDEX);
      at = min(max(at, 0), n_pos - 1);
    }
    turn = tab + (int64_t)at * half;
  }
  const int v0 = blockIdx.y * (kPgThreads / TPV) + (int)threadIdx.x / TPV;
  const int e0 = (int)threadIdx.x % TPV * 8;
  const int first = q_out ? 0 : p.Hq;
  for (int h0 = first; h0 < heads; h0 += gridDim.y * (kPgThreads / TPV)) {
    const int h = h0 + v0;
    const bool live = h < heads;
    float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const T* src = qkv + (row * heads + h) * HD;
    if (live) {
      if (h < p.Hq + p.Hkv && half > 0) turned8(src, e0, half, turn, f);
      else load8(src + e0, f);
    }
    if (live && h < p.Hq) store8(q_out + (row * p.Hq + h) * HD + e0, f);
    const bool cached = live && h >= p.Hq && page >= 0;
    const bool value = h >= p.Hq + p.Hkv;
    const int g = h - p.Hq - (value ? p.Hkv : 0);
    const int64_t vec = cached ? paged_vec(p, page, place, g) : 0;
    if (!I8) {
      if (cached) store8(static_cast<T*>(value ? p.v : p.k) + vec * HD + e0, f);
    } else {
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
      for (int o = 1; o < TPV; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      if (cached) {
        const float most = __uint_as_float(m);
        const bool bad = m >= 0x7f800000u, none = most < kPgTiny;
        const float scale = bad ? NAN : none ? 0.f : __fdiv_rn(most, 127.f);
        const float inv = bad || none ? 0.f : __fdiv_rn(127.f, most);
        uint32_t w[2] = {0, 0};
        if (!bad && !none) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            w[i >> 2] |= (uint32_t)(__float2int_rn(__fmul_rn(f[i], inv)) & 0xff) << (8 * (i & 3));
        }
        *reinterpret_cast<uint2*>(static_cast<int8_t*>(value ? p.v : p.k) + vec * HD + e0) = make_uint2(w[0], w[1]);
        if (e0 == 0) (value ? p.vs : p.ks)[vec] = scale;
      }
    }
  }
}

template <typename T, int HD, bool I8>
__global__ void __launch_bounds__(kPgThreads)
    paged_read_kernel(const Paged p, T* k_out, T* v_out, int* err) {
  constexpr int TPV = HD / 8;
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 31;
  const int b = paged_find(p, row, lane);
  int place = -1, page = -1;
  if (b < p.B) {
    const PagedSeq s = paged_seq(p, b, err);
    const int i = (int)(row - s.row0);
    if (i >= 0 && i < s.n) place = s.len - s.n + i;
    if (place >= 0) page = paged_page(p, b, place, err);
  }
  const int e0 = (int)threadIdx.x % TPV * 8;
  for (int h = (int)threadIdx.x / TPV; h < 2 * p.Hkv; h += kPgThreads / TPV) {
    const bool value = h >= p.Hkv;
    const int g = h - (value ? p.Hkv : 0);
    float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (page >= 0) {
      const int64_t vec = paged_vec(p, page, place, g);
      if (I8) {
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(value ? p.v : p.k) + vec * HD + e0);
        const float scale = (value ? p.vs : p.ks)[vec];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          f[i] = (float)(int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3))) * scale;
      } else {
        load8(static_cast<const T*>(value ? p.v : p.k) + vec * HD + e0, f);
      }
    }
    store8((value ? v_out : k_out) + (row * p.Hkv + g) * HD + e0, f);
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

cudaError_t paged_append(int dtype, const Paged& p, const void* qkv, const float2* tab, int half, int n_pos,
                         const int32_t* pos, void* q_out, const Dev& dev) {
  return with_kind(dtype, p, [&](auto t, auto hd, auto i8) -> cudaError_t {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    constexpr int per = kPgThreads / (HD / 8);
    const int vecs = (q_out ? p.Hq : 0) + 2 * p.Hkv;
    return launch_pdl(paged_append_kernel<T, HD, decltype(i8)::value>, dim3((unsigned)p.n_rows, (vecs + per - 1) / per),
                      dim3(kPgThreads), 0, dev.stream, p, static_cast<const T*>(qkv), tab, half, n_pos, pos,
                      static_cast<T*>(q_out), dev.err);
  });
}

cudaError_t paged_read(int dtype, const Paged& p, void* k_out, void* v_out, const Dev& dev) {
  return with_kind(dtype, p, [&](auto t, auto hd, auto i8) -> cudaError_t {
    using T = decltype(t);
    return launch_pdl(paged_read_kernel<T, decltype(hd)::value, decltype(i8)::value>, dim3((unsigned)p.n_rows),
                      dim3(kPgThreads), 0, dev.stream, p, static_cast<T*>(k_out), static_cast<T*>(v_out), dev.err);
  });
}

}  // namespace adadsf
