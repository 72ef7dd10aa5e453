// Embedding rows with a scale, and the gradient of the table.
//   y_i = s E[id_i],   dE[v] = s sum of dy_i over id_i = v
//
// Backward: the tokens are sorted by id (equal ones by place), then summed along the sorted list: a group of
// threads walks a run of places, adds the rows of one id in fp32 and writes an id's row when all of its places are
// its own. Sums of ids that go over a border are left beside the table and joined in order, so that a
// token that makes up a tenth of the batch is shared by many groups. Nothing depends on the order in which
// blocks run. Sorting: every token counts the ones before it where there are few (n^2 comparisons in one launch,
// no barrier), else digits of up to 9 bits, least first (three launches each: counts of a tile, their
// running sums, stable placing). The table's zeros are written by further blocks of the sort's launches, which leave the
// memory idle; rows of tokens that came are written again by the sums.
//
// Bound by memory where there are many tokens: 65536 tokens, a table of 152064 x 3584 bf16: rows 99 us, the sort with the table's 1.09 GB of
// zeros 172 (6.3 TB/s), sums 100, joins 13; in all 390. By the chain of launches where there are few: 100 tokens, 50304 x 768: 5, 12, 5 and
// 5 us one by one.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace adadsf {
namespace {

constexpr int kEgThreads = 512;     // at most, of a block
constexpr int kEgFew = 4096;        // tokens up to which each counts the ones before it
constexpr int kEgLanes = 16;        // lanes that share a token's count
constexpr int kEgFewThreads = 128;
constexpr int kEgSort = 256;        // threads of the digit sort
constexpr int kEgChunk = kEgSort * 8;
constexpr int kEgMaxTiles = 512;
constexpr int kEgDigit = 9;
constexpr int kEgAhead = 8;         // rows on their way

// Ids of no row of the table: below 0 padding, past it an error; both sort behind every id.
__device__ __forceinline__ int32_t key_of(int32_t id, int vocab, int* err) {
  if (id >= 0 && id < vocab) return id;
  if (id >= vocab) set_device_error(err, DEVERR_INDEX);
  return vocab;
}

template <typename T>
__global__ void __launch_bounds__(256)
    embed_scale_kernel(const int32_t* ids, int64_t n, const T* table, int vocab, int d, float scale, T* out, int* err) {
  pdl_wait();
  pdl_trigger();
  constexpr int V = Elem<T>::kVec;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= n) return;
  const int32_t id = ids[row];
  const bool ok = id >= 0 && id < vocab;
  if (id >= vocab && lane == 0) set_device_error(err, DEVERR_INDEX);
  const T* src = table + (int64_t)(ok ? id : 0) * d;
  T* dst = out + row * d;
  const int nv = d / V;
#pragma unroll 4
  for (int c = lane; c < nv; c += 32) {
    float f[V];
    if (ok) load_vec(src + c * V, f);
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = ok ? f[j] * scale : 0.f;
    store_vec(dst + c * V, f);
  }
}

// A share of the table's zeros, for the blocks from `first` on of a sort's launch.
struct Zeros {
  uint4* at;
  int64_t n;          // 16-byte pieces
  int first;
};
__device__ __forceinline__ void write_zeros(const Zeros& z) {
  const int64_t step = (int64_t)(gridDim.x - z.first) * blockDim.x;
  for (int64_t i = (int64_t)(blockIdx.x - z.first) * blockDim.x + threadIdx.x; i < z.n; i += step) z.at[i] = make_uint4(0, 0, 0, 0);
}

__global__ void __launch_bounds__(kEgFewThreads)
    embed_rank_kernel(const int32_t* ids, int n, int vocab, int32_t* key, int32_t* place, const Zeros z, int* err) {
  __shared__ __align__(16) int32_t k[kEgFew];
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x >= z.first) return write_zeros(z);
  const int padded = (n + 3) & ~3;
  for (int i = threadIdx.x; i < padded; i += kEgFewThreads) k[i] = i < n ? key_of(ids[i], vocab, err) : INT32_MAX;
  __syncthreads();
  const int i = (blockIdx.x * kEgFewThreads + threadIdx.x) / kEgLanes, part = threadIdx.x % kEgLanes;
  const int32_t mine = i < n ? k[i] : 0;
  int rank = 0;
  for (int j = part * 4; j < padded; j += 4 * kEgLanes) {
    const int4 o = *reinterpret_cast<const int4*>(k + j);
    // before it: a smaller id, or the same one at an earlier place
    rank += (o.x < mine + (j < i)) + (o.y < mine + (j + 1 < i)) + (o.z < mine + (j + 2 < i)) + (o.w < mine + (j + 3 < i));
  }
#pragma unroll
  for (int s = 1; s < kEgLanes; s <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, s);
  if (i < n && part == 0) {
    key[rank] = mine;
    place[rank] = i;
  }
}

struct Digit {
  const int32_t *key_in, *place_in;   // place_in null: the ids as they came
  int32_t *key, *place;
  int64_t n, per_tile;                // a multiple of kEgChunk
  int tiles, shift, bits, vocab;
  int32_t* counts;                    // [1 << bits][tiles], then its running sums
};

__device__ __forceinline__ int32_t key_at(const Digit& q, int64_t i, int* err) {
  return q.place_in ? q.key_in[i] : key_of(q.key_in[i], q.vocab, err);
}

__global__ void __launch_bounds__(kEgSort) embed_count_kernel(const Digit q, const Zeros z, int* err) {
  __shared__ int32_t c[1 << kEgDigit];
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x >= z.first) return write_zeros(z);
  const int digits = 1 << q.bits;
  for (int i = threadIdx.x; i < digits; i += kEgSort) c[i] = 0;
  __syncthreads();
  const int64_t end = min(q.n, (blockIdx.x + 1) * q.per_tile);
  for (int64_t i = blockIdx.x * q.per_tile + threadIdx.x; i < end; i += kEgSort)
    atomicAdd(&c[(key_at(q, i, err) >> q.shift) & (digits - 1)], 1);
  __syncthreads();
  for (int i = threadIdx.x; i < digits; i += kEgSort) q.counts[(int64_t)i * q.tiles + blockIdx.x] = c[i];
}

// Running sums (exclusive) of all counts, by one block.
__global__ void __launch_bounds__(1024) embed_scan_kernel(int32_t* counts, int n, const Zeros z) {
  __shared__ int32_t sums[32];
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x >= z.first) return write_zeros(z);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t before = 0;
  for (int c = 0; c < n; c += 4096) {
    const int i = c + threadIdx.x * 4;
    int32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = i + j < n ? counts[i + j] : 0;
    const int32_t mine = v[0] + v[1] + v[2] + v[3];
    int32_t run = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t up = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += up;
    }
    if (lane == 31) sums[warp] = run;
    __syncthreads();
    int32_t base = before, all = 0;
    for (int w = 0; w < 32; ++w) {
      if (w < warp) base += sums[w];
      all += sums[w];
    }
    base += run - mine;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i + j < n) counts[i + j] = base;
      base += v[j];
    }
    before += all;
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kEgSort) embed_place_kernel(const Digit q, const Zeros z, int* err) {
  constexpr int W = kEgSort / 32;
  __shared__ int32_t base[1 << kEgDigit];        // where the tile's next token of a digit goes
  __shared__ int32_t c[W][1 << kEgDigit];        // a chunk's counts by warp, then what lies before the warp
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x >= z.first) return write_zeros(z);
  const int digits = 1 << q.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < digits; i += kEgSort) base[i] = q.counts[(int64_t)i * q.tiles + blockIdx.x];
  const int64_t begin = blockIdx.x * q.per_tile, end = min(q.n, begin + q.per_tile);
  for (int64_t chunk = begin; chunk < end; chunk += kEgChunk) {
    for (int i = threadIdx.x; i < W * digits; i += kEgSort) c[i / digits][i % digits] = 0;
    __syncthreads();
    // a warp has kEgChunk / W places in a row, 32 at a time
    int32_t key[8], rank[8];
    const int64_t first = chunk + warp * (kEgChunk / W) + lane;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t i = first + j * 32;
      const bool in = i < end;
      key[j] = in ? key_at(q, i, err) : -1;
      const int digit = in ? (key[j] >> q.shift) & (digits - 1) : digits;
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      const int before = __popc(same & ((1u << lane) - 1));
      int32_t had = 0;
      if (in && before == 0) {
        had = c[warp][digit];
        c[warp][digit] = had + __popc(same);
      }
      had = __shfl_sync(0xffffffffu, had, __ffs(same) - 1);
      rank[j] = had + before;
      __syncwarp();
    }
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += kEgSort) {
      int32_t at = base[i];
      for (int w = 0; w < W; ++w) {
        const int32_t here = c[w][i];
        c[w][i] = at;
        at += here;
      }
      base[i] = at;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t i = first + j * 32;
      if (i >= end) continue;
      const int32_t to = c[warp][(key[j] >> q.shift) & (digits - 1)] + rank[j];
      q.key[to] = key[j];
      q.place[to] = q.place_in ? q.place_in[i] : (int32_t)i;
    }
    __syncthreads();
  }
}

struct EgDev {
  const int32_t *key, *place;
  int64_t n, runs;
  int run;             // places of a run
  const void* dy;
  int vocab, d, group, groups, nv;
  float scale;
  void* out;
  int add;
  float* carry;        // [runs][2][d]: the sum of an id that began before, of one that goes on behind
};

template <typename T>
__device__ __forceinline__ void write_row(const EgDev& p, int64_t id, int c, float* s) {
  constexpr int V = Elem<T>::kVec;
  T* at = static_cast<T*>(p.out) + id * p.d + c * V;
#pragma unroll
  for (int j = 0; j < V; ++j) s[j] *= p.scale;
  if (p.add) {
    float old[V];
    load_vec(at, old);
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] += old[j];
  }
  store_vec(at, s);
}

template <int V>
__device__ __forceinline__ void put_carry(const EgDev& p, int64_t at, int c, const float (&s)[V]) {
  float* to = p.carry + at * p.d + c * V;
#pragma unroll
  for (int j = 0; j < V; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
}

// A group of threads: a run of places of the sorted list, its threads the vectors of a row (blockIdx.y: which of them).
template <typename T>
__global__ void __launch_bounds__(kEgThreads) embed_sum_kernel(const __grid_constant__ EgDev p) {
  constexpr int V = Elem<T>::kVec;
  pdl_wait();
  pdl_trigger();
  const int g = threadIdx.x / p.group, c = blockIdx.y * p.group + threadIdx.x - g * p.group, lane = threadIdx.x & 31;
  const int64_t run = (int64_t)blockIdx.x * p.groups + g;
  if (run >= p.runs) return;
  const bool mine = c < p.nv;
  const int64_t i0 = run * p.run, i1 = min(p.n, i0 + p.run);
  // 32 places at a time, a lane of each warp a place; the next ones are on their way
  int32_t key = i0 + lane < i1 ? p.key[i0 + lane] : p.vocab, place = i0 + lane < i1 ? p.place[i0 + lane] : 0;
  const int32_t before = i0 > 0 ? p.key[i0 - 1] : -1, behind = i1 < p.n ? p.key[i1] : -1;
  const uint4* dy = static_cast<const uint4*>(p.dy);
  int32_t id = __shfl_sync(0xffffffffu, key, 0);
  if (id >= p.vocab) return;
  bool began = id == before;   // the id's first place is another group's
  float s[V] = {};
  for (int64_t at = i0; at < i1; at += 32) {
    const int used = __popc(__ballot_sync(0xffffffffu, key < p.vocab));   // padding sorts last
    const int64_t ahead = at + 32 + lane;
    const int32_t next_key = ahead < i1 ? p.key[ahead] : p.vocab, next_place = ahead < i1 ? p.place[ahead] : 0;
    for (int i = 0; i < used; i += kEgAhead) {
      uint4 u[kEgAhead];
#pragma unroll
      for (int a = 0; a < kEgAhead; ++a) {
        const int32_t from = __shfl_sync(0xffffffffu, place, (i + a) & 31);
        u[a] = mine && i + a < used ? dy[(int64_t)from * p.nv + c] : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int a = 0; a < kEgAhead; ++a) {
        const int32_t now = __shfl_sync(0xffffffffu, key, (i + a) & 31);
        if (i + a >= used) break;
        if (now != id) {
          if (mine) {
            if (began) put_carry<V>(p, run * 2, c, s);
            else write_row<T>(p, id, c, s);
          }
          began = false;
          id = now;
#pragma unroll
          for (int j = 0; j < V; ++j) s[j] = 0.f;
        }
        float f[V];
        unpack16(u[a], f, T());
#pragma unroll
        for (int j = 0; j < V; ++j) s[j] += f[j];
      }
    }
    key = next_key;
    place = next_place;
  }
  if (!mine) return;
  if (began) put_carry<V>(p, run * 2, c, s);
  else if (id == behind) put_carry<V>(p, run * 2 + 1, c, s);
  else write_row<T>(p, id, c, s);
}

// The group whose places an id begins in and goes on behind adds up what the others left of it, in order.
template <typename T>
__global__ void __launch_bounds__(kEgThreads) embed_join_kernel(const __grid_constant__ EgDev p) {
  constexpr int V = Elem<T>::kVec;
  pdl_wait();
  pdl_trigger();
  const int g = threadIdx.x / p.group, c = blockIdx.y * p.group + threadIdx.x - g * p.group;
  const int64_t run = (int64_t)blockIdx.x * p.groups + g;
  if (run >= p.runs || c >= p.nv) return;
  const int64_t i0 = run * p.run, i1 = i0 + p.run;
  if (i1 >= p.n) return;
  const int32_t id = p.key[i1 - 1], behind = p.key[i1], first = p.key[i0], before = i0 > 0 ? p.key[i0 - 1] : -1;
  if (id >= p.vocab || behind != id || (first == id && before == id)) return;   // ends here, or began before
  float s[V];
  const float* at = p.carry + (run * 2 + 1) * p.d + c * V;
#pragma unroll
  for (int j = 0; j < V; j += 4) load4(at + j, s + j);
  // the runs behind that begin with the id, eight at a time: their sums lie at the first of their two places
  bool more = true;
  for (int64_t r = run + 1; more && r < p.runs; r += kEgAhead) {
    float f[kEgAhead][V];
    bool in[kEgAhead];
#pragma unroll
    for (int a = 0; a < kEgAhead; ++a) in[a] = r + a < p.runs && p.key[(r + a) * p.run] == id;
#pragma unroll
    for (int a = 0; a < kEgAhead; ++a) {
      if (!in[a]) continue;   // most ids go over one border: eight rows for each would be read for nothing
      const float* from = p.carry + (r + a) * 2 * p.d + c * V;
#pragma unroll
      for (int j = 0; j < V; j += 4) load4(from + j, f[a] + j);
    }
#pragma unroll
    for (int a = 0; a < kEgAhead; ++a) {
      more = more && in[a];
      if (!more) break;
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] += f[a][j];
    }
  }
  write_row<T>(p, id, c, s);
}

struct EgPlan {
  int64_t runs, per_tile;
  int run, tiles, bits, passes, digit;
};
constexpr int64_t kEgRuns = 32 * 2432, kEgLongRuns = 128 * 2432;   // a row's warps times rows from which runs are 32 and 128 places long
EgPlan plan(int64_t n, int vocab, int d) {
  n = std::max<int64_t>(n, 1);
  EgPlan q;
  // Long runs leave fewer sums beside the table; short ones give every SM some 16 warps (8 bf16 features a thread, and
  // as many for fp32, whose plan is the same).
  const int64_t warps = n * ((d / 8 + 31) / 32);
  q.run = warps >= kEgLongRuns ? 128 : warps >= kEgRuns ? 32 : 8;
  q.runs = (n + q.run - 1) / q.run;
  q.bits = 1;
  while (q.bits < 31 && ((int64_t)1 << q.bits) <= vocab) ++q.bits;   // keys 0 .. vocab
  q.passes = (q.bits + kEgDigit - 1) / kEgDigit;
  q.digit = (q.bits + q.passes - 1) / q.passes;
  q.per_tile = ((n + kEgMaxTiles - 1) / kEgMaxTiles + kEgChunk - 1) / kEgChunk * kEgChunk;
  q.tiles = (int)((n + q.per_tile - 1) / q.per_tile);
  return q;
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

template <typename T>
cudaError_t sums(const EgDev& p, const Dev& dev) {
  const dim3 grid((unsigned)((p.runs + p.groups - 1) / p.groups), (unsigned)((p.nv + p.group - 1) / p.group));
  const cudaError_t e = launch_pdl(embed_sum_kernel<T>, grid, dim3(p.group * p.groups), 0, dev.stream, p);
  if (e != cudaSuccess || p.runs == 1) return e;
  return launch_pdl(embed_join_kernel<T>, grid, dim3(p.group * p.groups), 0, dev.stream, p);
}

}  // namespace

cudaError_t embed_scale(int dtype, const int32_t* ids, int64_t n, const void* table, int vocab, int d, float scale, void* out,
                        const Dev& dev) {
  const dim3 grid((unsigned)((n + 7) / 8));
  if (dtype == kBF16)
    return launch_pdl(embed_scale_kernel<bf16>, grid, dim3(256), 0, dev.stream, ids, n, static_cast<const bf16*>(table), vocab,
                      d, scale, static_cast<bf16*>(out), dev.err);
  return launch_pdl(embed_scale_kernel<float>, grid, dim3(256), 0, dev.stream, ids, n, static_cast<const float*>(table), vocab, d,
                    scale, static_cast<float*>(out), dev.err);
}

// What any number of tokens up to n needs: fewer tokens may mean more of the short runs, and more tiles.
size_t embed_backward_scratch(int64_t n, int vocab, int d) {
  const EgPlan q = plan(n, vocab, d);
  int64_t runs = q.runs;
  const int64_t warps = (d / 8 + 31) / 32;   // of a row; a fp32 row of 4 features counts as none
  for (int64_t from : {kEgRuns, kEgLongRuns})
    if (warps > 0) runs = std::max(runs, plan(std::min(n, (from - 1) / warps), vocab, d).runs);   // the last ones with shorter runs
  const int64_t tiles = std::min<int64_t>(kEgMaxTiles, (std::max<int64_t>(n, 1) + kEgChunk - 1) / kEgChunk);
  return 4 * up256((size_t)n * 4) + up256((size_t)tiles * sizeof(int32_t) << q.digit) + up256((size_t)runs * 2 * d * 4);
}

cudaError_t embed_backward(int dtype, const int32_t* ids, const void* dy, int64_t n, int vocab, int d, float scale, void* out,
                           bool add, void* scratch, const Dev& dev) {
  const EgPlan q = plan(n, vocab, d);
  uint8_t* at = static_cast<uint8_t*>(scratch);
  auto take = [&](size_t bytes) {
    void* r = at;
    at += up256(bytes);
    return r;
  };
  int32_t* key[2];
  int32_t* place[2];
  for (int i = 0; i < 2; ++i) {
    key[i] = static_cast<int32_t*>(take((size_t)n * 4));
    place[i] = static_cast<int32_t*>(take((size_t)n * 4));
  }
  int32_t* counts = static_cast<int32_t*>(take((size_t)q.tiles * sizeof(int32_t) << q.digit));
  const int vec = dtype == kBF16 ? 8 : 4;
  // the table's zeros, in as many shares as the sort has launches
  const bool few = n <= kEgFew;
  const int64_t pieces = add ? 0 : (int64_t)vocab * (d / vec);
  const int launches = few ? 1 : 3 * q.passes;
  int launch = 0;
  auto zeros = [&](int first, int threads) {
    const int64_t a = pieces * launch / launches, b = pieces * (launch + 1) / launches;
    ++launch;
    Zeros z = {static_cast<uint4*>(out) + a, b - a, first};
    const int64_t blocks = std::min<int64_t>((b - a + 4 * threads - 1) / (4 * threads), (int64_t)dev.num_sms * 2048 / threads);
    return std::make_pair(z, (unsigned)(first + blocks));
  };
  cudaError_t e = cudaSuccess;
  int last = 0;
  if (few) {
    const auto [z, grid] = zeros((int)((n * kEgLanes + kEgFewThreads - 1) / kEgFewThreads), kEgFewThreads);
    e = launch_pdl(embed_rank_kernel, dim3(grid), dim3(kEgFewThreads), 0, dev.stream, ids, (int)n, vocab, key[0], place[0], z,
                   dev.err);
  } else {
    for (int pass = 0; pass < q.passes && e == cudaSuccess; ++pass) {
      Digit s = {};
      s.key_in = pass ? key[last] : ids;
      s.place_in = pass ? place[last] : nullptr;
      if (pass) last ^= 1;
      s.key = key[last];
      s.place = place[last];
      s.n = n;
      s.per_tile = q.per_tile;
      s.tiles = q.tiles;
      s.shift = pass * q.digit;
      s.bits = q.digit;
      s.vocab = vocab;
      s.counts = counts;
      const auto [z0, g0] = zeros(q.tiles, kEgSort);
      e = launch_pdl(embed_count_kernel, dim3(g0), dim3(kEgSort), 0, dev.stream, s, z0, dev.err);
      if (e != cudaSuccess) break;
      const auto [z1, g1] = zeros(1, 1024);
      e = launch_pdl(embed_scan_kernel, dim3(g1), dim3(1024), 0, dev.stream, counts, q.tiles << q.digit, z1);
      if (e != cudaSuccess) break;
      const auto [z2, g2] = zeros(q.tiles, kEgSort);
      e = launch_pdl(embed_place_kernel, dim3(g2), dim3(kEgSort), 0, dev.stream, s, z2, dev.err);
    }
  }
  if (e != cudaSuccess) return e;
  EgDev p = {};
  p.key = key[last];
  p.place = place[last];
  p.n = n;
  p.runs = q.runs;
  p.run = q.run;
  p.dy = dy;
  p.vocab = vocab;
  p.d = d;
  p.nv = d / vec;
  p.group = std::min((p.nv + 31) / 32 * 32, kEgThreads);
  p.groups = std::max(1, 256 / p.group);
  p.scale = scale;
  p.out = out;
  p.add = add;
  p.carry = static_cast<float*>(take((size_t)q.runs * 2 * d * 4));
  return dtype == kBF16 ? sums<bf16>(p, dev) : sums<float>(p, dev);
}

}  // namespace adadsf
