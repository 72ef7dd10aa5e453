// Attention of new tokens over a paged cache: a warp per (row, query head), the lanes
// splitting the head, walks the visible keys with an online softmax in fp32.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace adadsf {
namespace {

constexpr int kPaThreads = 128;
constexpr int kPaFewRows = 64;   // packed rows of a sequence up to which paged_rows.cu runs

template <typename T, int HD, bool I8>
__global__ void __launch_bounds__(kPaThreads)
    paged_attention_kernel(const Paged p, const T* q, int64_t ld_q, T* out, float scale, int* err) {
  constexpr int PL = HD / 32;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (kPaThreads / 32) + (threadIdx.x >> 5);
  if (w >= p.n_rows * p.Hq) return;
  const int64_t row = w / p.Hq;
  const int h = (int)(w % p.Hq), g = h / (p.Hq / p.Hkv);
  const int b = paged_find(p, row, lane);
  int visible = 0;
  if (b < p.B) {
    const PagedSeq s = paged_seq(p, b, err);
    const int i = (int)(row - s.row0);
    if (i >= 0 && i < s.n) visible = s.len - s.n + i + 1;
  }
  float qv[PL], o[PL];
#pragma unroll
  for (int e = 0; e < PL; ++e) {
    qv[e] = Elem<T>::to_f(q[row * ld_q + (int64_t)h * HD + lane + 32 * e]) * scale;
    o[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  int page = -1;
  for (int j = 0; j < visible; ++j) {
    if ((j & ((1 << p.page_log2) - 1)) == 0) page = paged_page(p, b, j, err);
    float kf[PL], vf[PL], ks = 1.f, vs = 1.f;
    if (page >= 0) {
      const int64_t vec = paged_vec(p, page, j, g);
      if (I8) {
        ks = p.ks[vec];
        vs = p.vs[vec];
      }
#pragma unroll
      for (int e = 0; e < PL; ++e) {
        if (I8) {
          kf[e] = (float)static_cast<const int8_t*>(p.k)[vec * HD + lane + 32 * e];
          vf[e] = (float)static_cast<const int8_t*>(p.v)[vec * HD + lane + 32 * e];
        } else {
          kf[e] = Elem<T>::to_f(static_cast<const T*>(p.k)[vec * HD + lane + 32 * e]);
          vf[e] = Elem<T>::to_f(static_cast<const T*>(p.v)[vec * HD + lane + 32 * e]);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < PL; ++e) kf[e] = vf[e] = 0.f;
    }
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < PL; ++e) d = fmaf(qv[e], kf[e], d);
    const float sc = warp_sum(d) * ks;
    const float m_new = fmaxf(m, sc);
    const float base = m_new == -INFINITY ? 0.f : m_new;
    const float a = expf(m - base), pr = expf(sc - base);
    l = l * a + pr;
#pragma unroll
    for (int e = 0; e < PL; ++e) o[e] = o[e] * a + pr * vs * vf[e];
    m = m_new;
  }
#pragma unroll
  for (int e = 0; e < PL; ++e)
    out[(row * p.Hq + h) * HD + lane + 32 * e] = Elem<T>::from_f(visible > 0 ? o[e] / l : 0.f);
}

}  // namespace

size_t paged_attention_scratch(int dtype, const Paged& p) { return dtype == kBF16 ? std::max(paged_rows_scratch(p), paged_tc_scratch(p)) : 0; }

cudaError_t paged_attention(int dtype, const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch,
                            const Dev& dev) {
  if (dtype == kBF16 && (int64_t)p.max_new * (p.Hq / p.Hkv) <= kPaFewRows)
    return paged_rows(p, q, ld_q, out, sync, scratch, dev);
  if (dtype == kBF16 && paged_tc_takes(p)) return paged_tc(p, q, ld_q, out, sync, scratch, dev);
  const int64_t blocks = (p.n_rows * p.Hq + kPaThreads / 32 - 1) / (kPaThreads / 32);
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  auto run = [&](auto t, auto hd, auto i8) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    return launch_pdl(paged_attention_kernel<T, HD, decltype(i8)::value>, dim3((unsigned)blocks), dim3(kPaThreads), 0,
                      dev.stream, p, static_cast<const T*>(q), ld_q, static_cast<T*>(out), 1.f / sqrtf((float)HD), dev.err);
  };
  auto with_hd = [&](auto t, auto i8) {
    return p.hd == 128 ? run(t, std::integral_constant<int, 128>(), i8) : run(t, std::integral_constant<int, 64>(), i8);
  };
  if (dtype == kBF16) return p.i8 ? with_hd(bf16(), std::true_type()) : with_hd(bf16(), std::false_type());
  return p.i8 ? with_hd(0.f, std::true_type()) : with_hd(0.f, std::false_type());
}

}  // namespace adadsf
