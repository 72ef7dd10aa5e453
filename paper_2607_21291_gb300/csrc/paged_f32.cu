// Attention of new tokens over a paged cache, fp32 models (adadsf_paged_attention): CUDA cores, exact
// fp32 online softmax.
//
// 64 or 16 packed rows (token i's G query heads of a key/value head side by side, row i G + g)
// against tiles of 64 keys. A warp owns a quarter of the rows, so row maxima and sums are shuffles and
// weights pass through the warp's own part of shared memory. Scores: a thread has 8 rows x 4 keys, or 4 x 2
// of the smaller tile, operands read four features at a time from padded rows; P V: the same rows by its
// share of the features. Shared memory bounds either product (12 reads of 16 bytes for 128 multiply-adds;
// the smaller tile 6 for 32, for calls that reading the cache bounds). The next K tile loads during the softmax and
// P V, the next V tile during the scores: by asynchronous copies, or 8-bit numbers through
// registers, times their scales. Items lie on a line cut into equal pieces (PagedLine); pieces of a cut item leave partials that
// the one which finishes last joins in order.
// Keys that a row does not see are left out of its sums altogether: their weight is 0, but 0 times an infinity is not.
// Measured, 8 heads of 64: 4 x 600 tokens on 1000 cached 203 us, 31 TFLOP/s of the 74 that fp32 can (schedulers 65% busy,
// three quarters of that multiply-adds; two multiply-adds an instruction took 217 us, for the copies that make the
// weights pairs); 3 x 129 on 511 35 us; 8 single tokens on 4000 36 us, 3.6 TB/s.
// From 8-bit caches 213, 36 and 38 us.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace adadsf {
namespace {

constexpr int kPfTK = 64;                // keys of a tile
constexpr int kPfThreads = 128;
constexpr int kPfPLd = kPfTK + 4;
constexpr int kPfSms = 160;

template <int HD, int RT, bool I8>
struct PfCfg {
  static constexpr int TX = RT == 64 ? 16 : 32;       // threads along the keys
  static constexpr int NR = RT == 64 ? 8 : 4;         // rows of a thread
  static constexpr int KC = kPfTK / TX;               // keys of a thread
  static constexpr int NF = HD / TX;                  // output features of a thread: 2, 4 or 8
  static constexpr int LD = HD + 4;
  static constexpr int FLOATS = (RT + kPfTK) * LD + kPfTK * HD + RT * kPfPLd;
  static constexpr int SMEM = FLOATS * 4;
  static constexpr int PER_SM = RT == 64 ? (HD == 64 ? 2 : 1) : HD == 64 ? (I8 ? 3 : 4) : 2;   // as registers and shared memory allow
  static constexpr int PART = RT * HD + 2 * RT;       // floats of a partial: O a thread, then (m, l) a row
};

template <int RT>
struct PfCut {
  static constexpr int KEYS = kPfTK, PAD = 1, WHOLE = 4;
  int G;
  __device__ __forceinline__ int groups(int n) const { return (int)(((int64_t)n * G + RT - 1) / RT); }
  __device__ __forceinline__ int tokens(int g) const { return (int)((((int64_t)g + 1) * RT - 1) / G) + 1; }
};

template <int HD, int RT, bool I8>
__global__ void __launch_bounds__(kPfThreads)
    paged_f32_kernel(const Paged p, const float* q, int64_t ld_q, float* out, float scale, int* sync, float* parts, int* err) {
  using C = PfCfg<HD, RT, I8>;
  using Cut = PfCut<RT>;
  constexpr int TX = C::TX, NR = C::NR, KC = C::KC, NF = C::NF, RPW = RT / 4;
  extern __shared__ __align__(16) float smem_pf[];
  __shared__ int done_s;
  float* sQ = smem_pf;
  float* sK = sQ + RT * C::LD;
  float* sV = sK + kPfTK * C::LD;
  float* sP = sV + kPfTK * HD;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, tx = lane % TX;
  const int G = p.Hq / p.Hkv;
  auto row_of = [&](int i) { return warp * RPW + lane / TX + (32 / TX) * i; };
  pdl_wait();
  pdl_trigger();
  PagedLine<Cut> line{Cut{G}};
  int64_t per, ua, ub;
  line.piece(p, Cut::PAD + 2, (int)blockIdx.x, (int)gridDim.x, lane, err, &per, &ua, &ub);
  for (int64_t u = ua; u < ub;) {
    const PagedItem<Cut> it = line.item(p, &u, lane, err);
    int t0, t1;
    it.in(ua, ub, &t0, &t1);
    if (t0 >= t1) continue;
    const int x0 = it.grp * RT;                        // first packed row of the sequence
    int lim[NR];                                       // keys that the thread's rows see; -1: no row
    bool any = false;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int x = x0 + row_of(i), tok = x / G;
      lim[i] = tok < it.n ? max(0, it.len - it.n + tok + 1) : -1;
      any |= lim[i] >= 0;
    }
    any = __any_sync(0xffffffffu, any);                // a warp without rows only helps with loads
    const int open = it.len - it.n + x0 / G + 1;       // keys that every row of the item sees
    const int32_t* tab = p.table + (int64_t)it.b * p.max_pages;
    // where tile j's runs of 16 keys begin, as vector numbers: lane l has run l % 4 (-1: nowhere)
    auto runs_of = [&](int j) -> int64_t {
      const int place = j * kPfTK + (lane & 3) * 16;
      if (place >= it.seen) return -1;
      const int page = tab[place >> p.page_log2];
      if ((unsigned)page < (unsigned)p.n_pages) return paged_vec(p, page, place, it.h);
      set_device_error(err, DEVERR_INDEX);
      return -1;
    };
    // number of key r's vector of the tile (all lanes), or -1: nowhere, or past the last visible key
    auto vec_of = [&](int64_t runs, int j, int r) -> int64_t {
      const int64_t run = __shfl_sync(0xffffffffu, runs, r >> 4);
      return run >= 0 && j * kPfTK + r < it.seen ? run + (r & 15) : -1;
    };
    // 64 keys (or values) of tile j: fp32, asynchronous; others become zeros
    auto load_tile = [&](float* dst, int ld, const void* pool, int64_t runs, int j) {
      if (!I8) {
#pragma unroll 4
        for (int v = tid; v < kPfTK * HD / 4; v += kPfThreads) {
          const int r = v / (HD / 4), c = v % (HD / 4) * 4;
          const int64_t vec = vec_of(runs, j, r);
          cp_async16(smem_u32(dst + r * ld + c), static_cast<const float*>(pool) + (vec >= 0 ? vec * HD + c : 0), vec >= 0);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // 8-bit: a thread's 16 numbers at a time, into registers and later times their scale into shared memory
    constexpr int NV = kPfTK * HD / 16 / kPfThreads;
    uint4 raw[2][I8 ? NV : 1];
    float sc[2][I8 ? NV : 1];
    auto fetch = [&](int w, const void* pool, const float* scales, int64_t runs, int j) {
#pragma unroll
      for (int i = 0; i < (I8 ? NV : 0); ++i) {
        const int v = i * kPfThreads + tid, r = v / (HD / 16), c = v % (HD / 16);
        const int64_t vec = vec_of(runs, j, r);
        raw[w][i] = vec >= 0 ? *reinterpret_cast<const uint4*>(static_cast<const int8_t*>(pool) + vec * HD + 16 * c) : make_uint4(0, 0, 0, 0);
        sc[w][i] = vec >= 0 ? scales[vec] : 0.f;
      }
    };
    auto put = [&](int w, float* dst, int ld) {
#pragma unroll
      for (int i = 0; i < (I8 ? NV : 0); ++i) {
        const int v = i * kPfThreads + tid, r = v / (HD / 16), c = v % (HD / 16);
        const uint32_t in[4] = {raw[w][i].x, raw[w][i].y, raw[w][i].z, raw[w][i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float f[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = (float)(int8_t)(in[k] >> (8 * e)) * sc[w][i];
          store_vec(dst + r * ld + 16 * c + 4 * k, f);
        }
      }
    };
    // the item's queries (rows of none: zeros)
    for (int v = tid; v < RT * HD / 4; v += kPfThreads) {
      const int r = v / (HD / 4), c = v % (HD / 4) * 4, x = x0 + r, tok = x / G;
      const bool is = tok < it.n;
      cp_async16(smem_u32(sQ + r * C::LD + c), q + (is ? (it.row0 + tok) * ld_q + (int64_t)(it.h * G + x - tok * G) * HD + c : 0), is);
    }
    int64_t runs = runs_of(t0);
    load_tile(sK, C::LD, p.k, runs, t0);
    load_tile(sV, HD, p.v, runs, t0);
    if (I8) {
      fetch(0, p.k, p.ks, runs, t0);
      fetch(1, p.v, p.vs, runs, t0);
      put(0, sK, C::LD);
      put(1, sV, HD);
    }
    float m[NR], l[NR], o[NR][NF];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < NF; ++c) o[i][c] = 0.f;
    }
    // O += P V; MASKED: some row does not see some key of the tile
    auto pv = [&](auto masked_c, int j) {
      constexpr bool MASKED = decltype(masked_c)::value;
#pragma unroll 2
      for (int k = 0; k < kPfTK; k += 4) {
        float4 pr[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) pr[i] = *reinterpret_cast<const float4*>(sP + row_of(i) * kPfPLd + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v[NF];
          if (NF == 2) {
            const float2 t = *reinterpret_cast<const float2*>(sV + (k + e) * HD + 2 * tx);
            v[0] = t.x;
            v[1] = t.y;
          } else {
#pragma unroll
            for (int c = 0; c < NF; c += 4) load4(sV + (k + e) * HD + c * TX + 4 * tx, v + c);
          }
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            const float w = e == 0 ? pr[i].x : e == 1 ? pr[i].y : e == 2 ? pr[i].z : pr[i].w;
            if (!MASKED || j * kPfTK + k + e < lim[i])
#pragma unroll
              for (int c = 0; c < NF; ++c) o[i][c] = fmaf(w, v[c], o[i][c]);
          }
        }
      }
    };
    for (int j = t0; j < t1; ++j) {
      if (j + 1 < t1) runs = runs_of(j + 1);
      asm volatile("cp.async.wait_group 1;" ::: "memory");   // K of this tile (and Q); V may be on its way
      __syncthreads();
      if (I8 && j + 1 < t1) {
        fetch(0, p.k, p.ks, runs, j + 1);
        fetch(1, p.v, p.vs, runs, j + 1);
      }
      float s[NR][KC];
      if (any) {
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int c = 0; c < KC; ++c) s[i][c] = 0.f;
#pragma unroll 2
        for (int k = 0; k < HD; k += 4) {
          float4 kv[KC];
#pragma unroll
          for (int c = 0; c < KC; ++c) kv[c] = *reinterpret_cast<const float4*>(sK + (tx + TX * c) * C::LD + k);
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            const float4 a = *reinterpret_cast<const float4*>(sQ + row_of(i) * C::LD + k);
#pragma unroll
            for (int c = 0; c < KC; ++c)
              s[i][c] = fmaf(a.w, kv[c].w, fmaf(a.z, kv[c].z, fmaf(a.y, kv[c].y, fmaf(a.x, kv[c].x, s[i][c]))));
          }
        }
      }
      __syncthreads();   // K is read: the next tile's may land
      if (j + 1 < t1) {
        load_tile(sK, C::LD, p.k, runs, j + 1);
        put(0, sK, C::LD);
      } else {
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      const bool masked = (j + 1) * kPfTK > open;
      if (any) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          float mx = -INFINITY;
#pragma unroll
          for (int c = 0; c < KC; ++c) {
            s[i][c] *= scale;
            if (masked && j * kPfTK + tx + TX * c >= lim[i]) s[i][c] = -INFINITY;
            mx = fmaxf(mx, s[i][c]);
          }
#pragma unroll
          for (int b = TX / 2; b > 0; b >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, b));
          const float m_new = fmaxf(m[i], mx), base = m_new == -INFINITY ? 0.f : m_new;
          const float a = expf(m[i] - base);
          float sum = 0.f;
#pragma unroll
          for (int c = 0; c < KC; ++c) {
            const float w = expf(s[i][c] - base);
            sum += w;
            sP[row_of(i) * kPfPLd + tx + TX * c] = w;
          }
#pragma unroll
          for (int b = TX / 2; b > 0; b >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, b);
          l[i] = l[i] * a + sum;
          m[i] = m_new;
#pragma unroll
          for (int c = 0; c < NF; ++c) o[i][c] *= a;
        }
      }
      asm volatile("cp.async.wait_group 1;" ::: "memory");   // V of this tile
      __syncthreads();                                        // for all; P is the warp's own
      if (any) {
        if (masked) pv(std::true_type(), j);
        else pv(std::false_type(), j);
      }
      __syncthreads();   // V is read
      if (j + 1 < t1) {
        load_tile(sV, HD, p.v, runs, j + 1);
        put(1, sV, HD);
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    // ---- the piece's result: out, or a partial
    const int first = it.first_cta(per), last = it.last_cta(per, it.tiles - 1);
    if (first != last) {
      auto part_of = [&](int cta) { return parts + ((int64_t)cta * 2 + (cta == first ? 1 : 0)) * C::PART; };
      float* po = part_of((int)blockIdx.x);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
#pragma unroll
        for (int c = 0; c < NF; ++c) __stcg(po + (i * NF + c) * kPfThreads + tid, o[i][c]);
        if (tx == 0) __stcg(reinterpret_cast<float2*>(po + RT * HD) + row_of(i), make_float2(m[i], l[i]));
      }
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        done_s = atomicAdd(sync + first, 1) == last - first;
        if (done_s) sync[first] = 0;
        __threadfence();
      }
      __syncthreads();
      const bool done = done_s != 0;
      __syncthreads();   // read before the next item's
      if (!done) continue;
      __threadfence();
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < NF; ++c) o[i][c] = 0.f;
      }
      // maxima first: the sums of one piece then wait for no other's, and loads of several are in flight
#pragma unroll 4
      for (int cta = first; cta <= last; ++cta)
#pragma unroll
        for (int i = 0; i < NR; ++i) m[i] = fmaxf(m[i], __ldcg(reinterpret_cast<const float2*>(part_of(cta) + RT * HD) + row_of(i)).x);
#pragma unroll 2
      for (int cta = first; cta <= last; ++cta) {
        const float* po2 = part_of(cta);
        float x[NR][NF];
        float2 ml[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          ml[i] = __ldcg(reinterpret_cast<const float2*>(po2 + RT * HD) + row_of(i));
#pragma unroll
          for (int c = 0; c < NF; ++c) x[i][c] = __ldcg(po2 + (i * NF + c) * kPfThreads + tid);
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          const float f = expf(ml[i].x - (m[i] == -INFINITY ? 0.f : m[i]));
          l[i] += ml[i].y * f;
#pragma unroll
          for (int c = 0; c < NF; ++c) o[i][c] += x[i][c] * f;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      if (lim[i] < 0) continue;
      const int x = x0 + row_of(i), tok = x / G;
      float* dst = out + ((it.row0 + tok) * p.Hq + it.h * G + x - tok * G) * HD;
      float v[NF];
#pragma unroll
      for (int c = 0; c < NF; ++c) v[c] = lim[i] > 0 ? o[i][c] / l[i] : 0.f;
      if (NF == 2) {
        *reinterpret_cast<float2*>(dst + 2 * tx) = make_float2(v[0], v[1]);
      } else {
#pragma unroll
        for (int c = 0; c < NF; c += 4) store_vec(dst + c * TX + 4 * tx, v + c);
      }
    }
    __syncthreads();   // shared memory is free for the next item
  }
}

template <int HD, int RT, bool I8>
cudaError_t launch_f32(const Paged& p, const float* q, int64_t ld_q, float* out, int* sync, float* scratch, const Dev& dev) {
  using C = PfCfg<HD, RT, I8>;
  const cudaError_t e = allow_smem<paged_f32_kernel<HD, RT, I8>, C::SMEM>();
  if (e != cudaSuccess) return e;
  const int G = p.Hq / p.Hkv;
  const int64_t span = ((int64_t)p.max_pages << p.page_log2) / kPfTK + 2;
  const int64_t groups = std::min<int64_t>((int64_t)p.B * ((p.max_new * (int64_t)G + RT - 1) / RT), p.n_rows * G);
  const int64_t most = std::max<int64_t>(1, groups * p.Hkv * span / 3 + 1);
  return launch_pdl(paged_f32_kernel<HD, RT, I8>, dim3((unsigned)std::min<int64_t>(most, (int64_t)std::min(dev.num_sms, kPfSms) * C::PER_SM)),
                    dim3(kPfThreads), (size_t)C::SMEM, dev.stream, p, q, ld_q, out, 1.f / sqrtf((float)HD), sync, scratch, dev.err);
}

template <int HD, int RT>
cudaError_t launch_f32_store(const Paged& p, const float* q, int64_t ld_q, float* out, int* sync, float* scratch, const Dev& dev) {
  return p.i8 ? launch_f32<HD, RT, true>(p, q, ld_q, out, sync, scratch, dev)
              : launch_f32<HD, RT, false>(p, q, ld_q, out, sync, scratch, dev);
}

template <int HD, int RT>
constexpr size_t f32_scratch() { return (size_t)kPfSms * PfCfg<HD, RT, false>::PER_SM * 2 * PfCfg<HD, RT, false>::PART * 4; }

}  // namespace

size_t paged_f32_scratch(const Paged& p) {
  return p.hd == 64 ? std::max(f32_scratch<64, 64>(), f32_scratch<64, 16>()) : std::max(f32_scratch<128, 64>(), f32_scratch<128, 16>());
}

cudaError_t paged_f32(const Paged& p, const void* q, int64_t ld_q, void* out, int* sync, void* scratch, const Dev& dev) {
  const float* qf = static_cast<const float*>(q);
  float *of = static_cast<float*>(out), *sf = static_cast<float*>(scratch);
  const bool few = (int64_t)p.max_new * (p.Hq / p.Hkv) <= 16;
  if (p.hd == 64)
    return few ? launch_f32_store<64, 16>(p, qf, ld_q, of, sync, sf, dev) : launch_f32_store<64, 64>(p, qf, ld_q, of, sync, sf, dev);
  return few ? launch_f32_store<128, 16>(p, qf, ld_q, of, sync, sf, dev) : launch_f32_store<128, 64>(p, qf, ld_q, of, sync, sf, dev);
}

}  // namespace adadsf
