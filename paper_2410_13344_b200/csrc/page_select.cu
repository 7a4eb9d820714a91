// The pages of a long cache that are worth reading for one new token, by an upper bound of what their keys can score:
//
//   score(page) = max over the query heads h of the KV head of  sum_d max(q[h][d] kmin[d], q[h][d] kmax[d])
//               = max_h  sum_d max(q, 0) kmax + min(q, 0) kmin,
//
// kmin and kmax the smallest and largest of the page's keys, element by element (cerb_kv_append keeps them): a sixteenth of the cache's bytes.
//
// The decisions are those of exact arithmetic, ties going to the lower page.  Scores are computed in fp32 together with a bound E of their error.
// A page further than 2 E above or below the border between the last one taken and the first one left is decided by that; the few in
// between are scored again in fp64.  (Summaries and queries of 16-bit elements: the products are exact in fp64 and their sums nearly always.)
#include <math.h>
#include <string.h>

#include <algorithm>

#include "cerb_internal.cuh"

namespace cerb {

namespace {

constexpr int SC_WARPS = 4;
constexpr int SEL_THREADS = 1024;
constexpr int SEL_BINS = 1024;
constexpr int SEL_LIST = 1024;              // pages near the border that are ranked one against another
constexpr int SEL_SMEM_PAGES = 40960;       // scores of up to this many pages lie in shared memory
constexpr int kMaxSelectPages = 1 << 17;    // (bit masks of them do always)

struct SelectParams {
  const void *q, *k_min, *k_max;
  const int32_t *page_table, *len;
  int32_t *sel, *n_sel;
  float *score, *bound;        // [unit][max_pages]; [unit][chunks]: the largest error bound of a chunk
  double* again;               // [unit][max_pages]
  long long q_row, q_head;     // elements
  int B, H, Hk, G, max_pages, n_pool_pages, K, n_first, n_last, chunks;
};

__device__ __forceinline__ int pages_held(const SelectParams& p, int b) {
  return (min(max(p.len[b], 0), p.max_pages * CERB_PAGE) + CERB_PAGE - 1) / CERB_PAGE;
}
__device__ __forceinline__ int page_at(const SelectParams& p, int b, int page) {
  const int at = p.page_table[(size_t)b * p.max_pages + page];
  return at >= 0 && at < p.n_pool_pages ? at : -1;
}

__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t abs2(uint32_t a) { return a & 0x7fff7fffu; }

// How far a score may be off, relative to S = sum_d |q_d| max(|kmin_d|, |kmax_d|).
// bf16: 2 Dh <= 256 products in steps of 16; a step of the tensor cores keeps at least 24 bits of the largest of its 17 addends, each of which is at most
// S: 16 steps of 17 x 2^-23 S, under 2^-14 S with S's own error.  fp32: sums of Dh products in chains of at most Dh / 32 + 5 roundings: under 2^-19 S.
template <typename T> __device__ __forceinline__ float error_factor();
template <> __device__ __forceinline__ float error_factor<bf16>() { return 1.0f / 16384; }
template <> __device__ __forceinline__ float error_factor<float>() { return 1.0f / 524288; }

// bf16 scores: 16 pages on the rows of a warp MMA, eight heads on its columns, kmax and kmin straight from global memory in the order in which the lanes
// load them.  The bound S is a third product.
template <int DH>
__global__ void __launch_bounds__(SC_WARPS * 32) page_score_bf16_kernel(const SelectParams p) {
  constexpr int KC = DH / 32, LD = DH + 8;
  extern __shared__ __align__(16) bf16 q_s[];                            // [heads padded to 8][LD]
  __shared__ float s_e[SC_WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int chunk = blockIdx.x % p.chunks, unit = blockIdx.x / p.chunks, kvh = unit % p.Hk, b = unit / p.Hk;
  griddep_wait();
  griddep_launch();
  const int N = pages_held(p, b);
  if (N <= p.K) return;                                                  // all of them
  const int tiles = (p.G + 7) / 8;
  for (int i = threadIdx.x; i < tiles * 8 * (DH / 8); i += SC_WARPS * 32) {
    const int h = i / (DH / 8), c = i % (DH / 8) * 8;
    *reinterpret_cast<uint4*>(q_s + h * LD + c) =
        h < p.G ? *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(p.q) + (size_t)b * p.q_row + (size_t)(kvh * p.G + h) * p.q_head + c)
                : make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  float bound = 0.f;
  for (int r = chunk * SC_WARPS + warp; r * 16 < N; r += p.chunks * SC_WARPS) {
    uint4 hi[2][KC], lo[2][KC];
    int at[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int page = r * 16 + g + 8 * e;
      at[e] = page < N ? page_at(p, b, page) : -1;
      const size_t from = ((size_t)max(at[e], 0) * p.Hk + kvh) * DH + 8 * t;
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        hi[e][j] = lo[e][j] = make_uint4(0, 0, 0, 0);
        if (at[e] >= 0) {
          hi[e][j] = *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(p.k_max) + from + 32 * j);
          lo[e][j] = *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(p.k_min) + from + 32 * j);
        }
      }
    }
    float best[2] = {-INFINITY, -INFINITY};
    bool nan[2] = {false, false};
    for (int n = 0; n < tiles; ++n) {
      float sh[4] = {0.f, 0.f, 0.f, 0.f}, sl[4] = {0.f, 0.f, 0.f, 0.f}, sb[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        const uint4 qv = *reinterpret_cast<const uint4*>(q_s + (8 * n + g) * LD + 32 * j + 8 * t);
        const uint32_t qw[4] = {qv.x, qv.y, qv.z, qv.w};
        const uint32_t h0[4] = {hi[0][j].x, hi[0][j].y, hi[0][j].z, hi[0][j].w}, h1[4] = {hi[1][j].x, hi[1][j].y, hi[1][j].z, hi[1][j].w};
        const uint32_t l0[4] = {lo[0][j].x, lo[0][j].y, lo[0][j].z, lo[0][j].w}, l1[4] = {lo[1][j].x, lo[1][j].y, lo[1][j].z, lo[1][j].w};
#pragma unroll
        for (int w = 0; w < 4; w += 2) {
          mma_16816(sh, h0[w], h1[w], h0[w + 1], h1[w + 1], max2(qw[w], 0u), max2(qw[w + 1], 0u));
          mma_16816(sl, l0[w], l1[w], l0[w + 1], l1[w + 1], min2(qw[w], 0u), min2(qw[w + 1], 0u));
          mma_16816(sb, max2(abs2(h0[w]), abs2(l0[w])), max2(abs2(h1[w]), abs2(l1[w])), max2(abs2(h0[w + 1]), abs2(l0[w + 1])),
                    max2(abs2(h1[w + 1]), abs2(l1[w + 1])), abs2(qw[w]), abs2(qw[w + 1]));
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (8 * n + 2 * t + (e & 1) >= p.G) continue;
        const float s = sh[e] + sl[e];
        nan[e >> 1] |= s != s;
        best[e >> 1] = fmaxf(best[e >> 1], s);
        if (at[e >> 1] >= 0) bound = sb[e] == sb[e] ? fmaxf(bound, sb[e]) : INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float s = nan[e] ? NAN : best[e];
#pragma unroll
      for (int w = 1; w < 4; w <<= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, s, w);
        s = s != s || other != other ? NAN : fmaxf(s, other);
      }
      const int page = r * 16 + g + 8 * e;
      // (a page that lies nowhere: below every other)
      if (t == 0 && page < N) p.score[(size_t)unit * p.max_pages + page] = at[e] >= 0 ? s : -INFINITY;
    }
  }
#pragma unroll
  for (int w = 1; w < 32; w <<= 1) bound = fmaxf(bound, __shfl_xor_sync(0xffffffffu, bound, w));
  if (lane == 0) s_e[warp] = bound;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < SC_WARPS; ++w) bound = fmaxf(bound, s_e[w]);
    p.bound[(size_t)unit * p.chunks + chunk] = bound * error_factor<bf16>();
  }
}

// fp32 scores: a page to a warp, DH / 32 elements to a lane.
template <int DH>
__global__ void __launch_bounds__(SC_WARPS * 32) page_score_f32_kernel(const SelectParams p) {
  constexpr int E = DH / 32;
  extern __shared__ __align__(16) float qf_s[];                          // [heads][DH]
  __shared__ float s_e[SC_WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunk = blockIdx.x % p.chunks, unit = blockIdx.x / p.chunks, kvh = unit % p.Hk, b = unit / p.Hk;
  griddep_wait();
  griddep_launch();
  const int N = pages_held(p, b);
  if (N <= p.K) return;
  for (int i = threadIdx.x; i < p.G * DH; i += SC_WARPS * 32)
    qf_s[i] = reinterpret_cast<const float*>(p.q)[(size_t)b * p.q_row + (size_t)(kvh * p.G + i / DH) * p.q_head + i % DH];
  __syncthreads();
  float bound = 0.f;
  for (int page = chunk * SC_WARPS + warp; page < N; page += p.chunks * SC_WARPS) {
    const int at = page_at(p, b, page);
    float hi[E], lo[E], best = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const size_t from = ((size_t)max(at, 0) * p.Hk + kvh) * DH + lane * E + e;
      hi[e] = at >= 0 ? reinterpret_cast<const float*>(p.k_max)[from] : 0.f;
      lo[e] = at >= 0 ? reinterpret_cast<const float*>(p.k_min)[from] : 0.f;
    }
    for (int h = 0; h < p.G; ++h) {
      float s = 0.f, a = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float x = qf_s[h * DH + lane * E + e];
        s = fmaf(x, x >= 0.f ? hi[e] : lo[e], s);
        a = fmaf(fabsf(x), fmaxf(fabsf(hi[e]), fabsf(lo[e])), a);
      }
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, w);
        a += __shfl_xor_sync(0xffffffffu, a, w);
      }
      nan |= s != s;
      best = fmaxf(best, s);
      bound = a == a ? fmaxf(bound, a) : INFINITY;
    }
    if (lane == 0) p.score[(size_t)unit * p.max_pages + page] = at < 0 ? -INFINITY : nan ? NAN : best;
  }
  if (lane == 0) s_e[warp] = bound;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < SC_WARPS; ++w) bound = fmaxf(bound, s_e[w]);
    p.bound[(size_t)unit * p.chunks + chunk] = bound * error_factor<float>();
  }
}

// A page's score in fp64, by a warp; a NaN ranks first.
template <typename T> __device__ __forceinline__ double wide(T x);
template <> __device__ __forceinline__ double wide<float>(float x) { return (double)x; }
template <> __device__ __forceinline__ double wide<bf16>(bf16 x) { return (double)__bfloat162float(x); }
template <typename T, int DH>
__device__ double score_again(const SelectParams& p, int b, int kvh, int page, int lane) {
  constexpr int E = DH / 32;
  const int at = page_at(p, b, page);
  if (at < 0) return -INFINITY;
  const T* hi = reinterpret_cast<const T*>(p.k_max) + ((size_t)at * p.Hk + kvh) * DH + lane;
  const T* lo = reinterpret_cast<const T*>(p.k_min) + ((size_t)at * p.Hk + kvh) * DH + lane;
  double h[E], l[E], best = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) { h[e] = wide<T>(hi[32 * e]); l[e] = wide<T>(lo[32 * e]); }
  for (int g = 0; g < p.G; ++g) {
    const T* q = reinterpret_cast<const T*>(p.q) + (size_t)b * p.q_row + (size_t)(kvh * p.G + g) * p.q_head + lane;
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double x = wide<T>(q[32 * e]), a = x * l[e], c = x * h[e];
      s += a != a || c != c ? a + c : fmax(a, c);
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
    best = s != s || best != best ? (double)NAN : fmax(best, s);
  }
  return best != best ? (double)INFINITY : best;
}

// Order-preserving images of floats and doubles.
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i >= 0 ? i : i ^ 0x7fffffff;
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i >= 0 ? i : i ^ 0x7fffffff); }
__device__ __forceinline__ unsigned long long ordered(double x) {
  if (x == 0.0) x = 0.0;                                                 // (one zero)
  const unsigned long long i = (unsigned long long)__double_as_longlong(x);
  return i >> 63 ? ~i : i | 0x8000000000000000ull;
}

__device__ __forceinline__ int block_sum(int v, int* red) {
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, red[threadIdx.x & 31]);
}
__device__ __forceinline__ int block_scan(int v, int* red, int& total) {     // exclusive
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  __syncthreads();
  if (lane == 31) red[warp] = s;
  __syncthreads();
  int w = red[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += u;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
  return s - v + (warp ? before : 0);
}

// One CTA per (sequence, KV head).  The border is closed in on by histograms between the smallest and the largest score (a bin is a range of values; a score's
// bin is a monotonic function of it), each level in the range of the bin that holds the border, until few pages are left in it; those, and
// what lies within 2 E of them, are ranked in fp64.
template <typename T, int DH>
__global__ void __launch_bounds__(SEL_THREADS, 1) page_select_kernel(const SelectParams p) {
  extern __shared__ __align__(16) float score_s[];
  __shared__ int red[32], hist[SEL_BINS];
  __shared__ unsigned taken[kMaxSelectPages / 32];
  __shared__ int list[SEL_LIST];
  __shared__ double again[SEL_LIST];
  __shared__ int s_lo, s_hi, s_n, s_bin, s_above;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, kvh = unit % p.Hk, b = unit / p.Hk;
  griddep_wait();
  griddep_launch();
  const int N = pages_held(p, b), n = min(N, p.K);
  int32_t* sel = p.sel + (size_t)unit * p.K;
  if (kvh == 0 && tid == 0) p.n_sel[b] = n;
  for (int i = n + tid; i < p.K; i += SEL_THREADS) sel[i] = -1;
  if (N <= p.K) {
    for (int i = tid; i < N; i += SEL_THREADS) sel[i] = i;
    return;
  }
  const int first = p.n_first, last = N - p.n_last;                      // pages first .. last - 1 are up for selection
  const int want = p.K - first - p.n_last;                               // (K >= n_first + n_last, and N > K)
  const int words = (N + 31) / 32;
  for (int i = tid; i < words; i += SEL_THREADS) {
    // the forced ones
    unsigned m = 0;
    for (int j = 0; j < 32; ++j) {
      const int page = i * 32 + j;
      if (page < N && (page < first || page >= last)) m |= 1u << j;
    }
    taken[i] = m;
  }
  if (tid == 0) { s_lo = ordered(INFINITY); s_hi = ordered(-INFINITY); s_n = 0; }
  float bound = 0.f;
  for (int i = tid; i < p.chunks; i += SEL_THREADS) bound = fmaxf(bound, p.bound[(size_t)unit * p.chunks + i]);
  __syncthreads();
  const float* score = p.score + (size_t)unit * p.max_pages;
  {
    float lo = INFINITY, hi = -INFINITY;
    int odd = 0;
    for (int i = first + tid; i < last; i += SEL_THREADS) {
      const float s = score[i];
      if (N <= SEL_SMEM_PAGES) score_s[i] = s;
      if (!(fabsf(s) < INFINITY)) ++odd;
      lo = fminf(lo, s);
      hi = fmaxf(hi, s);
    }
    const int l = __reduce_min_sync(0xffffffffu, ordered(lo)), h = __reduce_max_sync(0xffffffffu, ordered(hi));
    const int e = __reduce_max_sync(0xffffffffu, __float_as_int(bound));   // (not negative, not a NaN)
    if (lane == 0) { atomicMin(&s_lo, l); atomicMax(&s_hi, h); red[warp] = e; }
    odd = __reduce_add_sync(0xffffffffu, odd);
    if (lane == 0 && odd) atomicAdd(&s_n, odd);
  }
  __syncthreads();
  const float E = __int_as_float(__reduce_max_sync(0xffffffffu, red[lane]));
  if (N <= SEL_SMEM_PAGES) score = score_s;
  float lo = from_ordered(s_lo), hi = from_ordered(s_hi);
  const bool all_again = s_n > 0 || !(E < INFINITY);                     // scores that are not finite decide nothing
  int above = 0;                                                         // pages above hi
  float t_lo = -INFINITY, t_hi = INFINITY;
  if (!all_again && want > 0) {
    for (int level = 0; level < 8; ++level) {
      __syncthreads();
      for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[i] = 0;
      __syncthreads();
      const float inv = (float)SEL_BINS / (hi - lo);
      auto bin_of = [&](float s) { return min(SEL_BINS - 1, max(0, (int)((s - lo) * inv))); };
      if (!(hi > lo) || !(inv < INFINITY)) break;
      for (int i = first + tid; i < last; i += SEL_THREADS) {
        const float s = score[i];
        if (s >= lo && s <= hi) atomicAdd(&hist[bin_of(s)], 1);
      }
      __syncthreads();
      // the bin with the want-th best: thread i looks at the i-th bin from above
      static_assert(SEL_BINS == SEL_THREADS, "a bin per thread");
      const int mine = hist[SEL_BINS - 1 - tid];
      int total;
      const int before = above + block_scan(mine, red, total);
      if (before < want && before + mine >= want) { s_bin = SEL_BINS - 1 - tid; s_above = before; s_lo = ordered(INFINITY); s_hi = ordered(-INFINITY); }
      __syncthreads();
      const int bin = s_bin, count = hist[bin];
      float l = INFINITY, h = -INFINITY;
      for (int i = first + tid; i < last; i += SEL_THREADS) {
        const float s = score[i];
        if (s >= lo && s <= hi && bin_of(s) == bin) { l = fminf(l, s); h = fmaxf(h, s); }
      }
      const int lw = __reduce_min_sync(0xffffffffu, ordered(l)), hw = __reduce_max_sync(0xffffffffu, ordered(h));
      if (lane == 0) { atomicMin(&s_lo, lw); atomicMax(&s_hi, hw); }
      __syncthreads();
      above = s_above;
      lo = from_ordered(s_lo);
      hi = from_ordered(s_hi);
      if (count <= 32 || hi - lo <= E) break;
    }
    t_lo = lo - 2.1f * E;
    t_hi = hi + 2.1f * E;
  }
  // sure ones and those near the border
  __syncthreads();
  if (tid == 0) s_n = 0;
  __syncthreads();
  int sure = 0;
  if (want > 0)
    for (int i = first + tid; i < last; i += SEL_THREADS) {
      const float s = score[i];
      if (!all_again && s > t_hi) {
        atomicOr(&taken[i >> 5], 1u << (i & 31));
        ++sure;
      } else if (all_again || s >= t_lo) {
        const int at = atomicAdd(&s_n, 1);
        if (at < SEL_LIST) list[at] = i;
      }
    }
  sure = block_sum(sure, red);
  const int near = s_n, rest = want - sure;
  if (near == rest || near <= SEL_LIST) {
    if (near > rest) {
      for (int i = warp; i < near; i += SEL_THREADS / 32) {
        const double s = score_again<T, DH>(p, b, kvh, list[i], lane);
        if (lane == 0) again[i] = s;
      }
      __syncthreads();
      for (int i = tid; i < near; i += SEL_THREADS) {
        int rank = 0;
        for (int j = 0; j < near; ++j) rank += again[j] > again[i] || (again[j] == again[i] && list[j] < list[i]);
        if (rank < rest) atomicOr(&taken[list[i] >> 5], 1u << (list[i] & 31));
      }
    } else if (near <= SEL_LIST) {
      for (int i = tid; i < near; i += SEL_THREADS) atomicOr(&taken[list[i] >> 5], 1u << (list[i] & 31));
    } else {
      for (int i = first + tid; i < last; i += SEL_THREADS)
        if (all_again || score[i] >= t_lo) atomicOr(&taken[i >> 5], 1u << (i & 31));
    }
  } else {
    // many near the border (a cache of equal keys, scores that are not finite): all of them in fp64, the border by bisection of the ordered values
    double* far = p.again + (size_t)unit * p.max_pages;
    auto is_near = [&](int i) { return all_again || (score[i] >= t_lo && score[i] <= t_hi); };
    for (int i = first + warp; i < last; i += SEL_THREADS / 32)
      if (is_near(i)) {
        const double s = score_again<T, DH>(p, b, kvh, i, lane);
        if (lane == 0) far[i] = s;
      }
    __syncthreads();
    unsigned long long v = 0;                                            // the largest that `rest` or more are not below
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long c = v | 1ull << bit;
      int cnt = 0;
      for (int i = first + tid; i < last; i += SEL_THREADS) cnt += is_near(i) && ordered(far[i]) >= c;
      if (block_sum(cnt, red) >= rest) v = c;
    }
    int over = 0;
    for (int i = first + tid; i < last; i += SEL_THREADS)
      if (is_near(i) && ordered(far[i]) > v) {
        atomicOr(&taken[i >> 5], 1u << (i & 31));
        ++over;
      }
    int ties = rest - block_sum(over, red);
    for (int i0 = first; i0 < last && ties > 0; i0 += SEL_THREADS) {
      const int i = i0 + tid;
      const int tie = i < last && is_near(i) && ordered(far[i]) == v;
      int total;
      const int before = block_scan(tie, red, total);
      if (tie && before < ties) atomicOr(&taken[i >> 5], 1u << (i & 31));
      ties -= total;
    }
  }
  __syncthreads();
  int written = 0;
  for (int w0 = 0; w0 < words; w0 += SEL_THREADS) {
    unsigned m = w0 + tid < words ? taken[w0 + tid] : 0;
    int total, at = written + block_scan(__popc(m), red, total);
    for (; m; m &= m - 1) sel[at++] = (w0 + tid) * 32 + __ffs(m) - 1;
    written += total;
  }
}

int plan_select(int dtype, int B, int H, int Hk, int head_dim, int max_pages, size_t* score_bytes, size_t* bound_bytes, size_t* again_bytes, int max_len, int* chunks) {
  if (dtype != CERB_F32 && dtype != CERB_BF16) return CERB_E_ARG;
  if (B < 0 || H < 1 || Hk < 1 || H % Hk || (head_dim != 64 && head_dim != 128) || max_pages < 1 || max_pages > kMaxSelectPages) return CERB_E_SHAPE;
  if (H / Hk > 64 || (long long)B * Hk > 0x7fffffll) return CERB_E_SHAPE;
  const long long units = (long long)B * Hk;
  // CTAs for every SM a few times over, of no less than a round of their warps
  const int held = (int)(((long long)max_len + CERB_PAGE - 1) / CERB_PAGE), per = dtype == CERB_BF16 ? 16 * SC_WARPS : SC_WARPS;
  const long long most = (std::min(held, max_pages) + per - 1) / per, want = units ? (148 * 8 + units - 1) / units : 1;
  *chunks = (int)std::max(1ll, std::min(most, want));
  *score_bytes = ((size_t)units * max_pages * sizeof(float) + 255) & ~(size_t)255;
  *bound_bytes = ((size_t)units * *chunks * sizeof(float) + 255) & ~(size_t)255;
  *again_bytes = (size_t)units * max_pages * sizeof(double);
  return CERB_OK;
}

}  // namespace

}  // namespace cerb

using namespace cerb;

extern "C" {

int cerb_page_select_scratch_bytes(int32_t dtype, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_pages, int32_t max_len,
                                   size_t* bytes_out) {
  if (!bytes_out || max_len < 1) return CERB_E_ARG;
  size_t s, e, g;
  int chunks;
  CERB_TRY(plan_select(dtype, B, n_heads, n_kv_heads, head_dim, max_pages, &s, &e, &g, max_len, &chunks));
  *bytes_out = s + e + g;
  return CERB_OK;
}

int cerb_page_select(const cerb_page_select_args* a, void* stream) {
  if (!a || (a->B > 0 && (!a->q || !a->k_min || !a->k_max || !a->page_table || !a->len || !a->sel || !a->n_sel))) return CERB_E_ARG;
  if (a->n_pool_pages < 1 || a->max_len < 1 || a->n_first < 0 || a->n_last < 0 || a->max_sel < 1) return CERB_E_ARG;
  if ((long long)a->n_first + a->n_last > a->max_sel) return CERB_E_SHAPE;
  size_t s, e, g;
  int chunks;
  CERB_TRY(plan_select(a->dtype, a->B, a->n_heads, a->n_kv_heads, a->head_dim, a->max_pages, &s, &e, &g, a->max_len, &chunks));
  const int es = a->dtype == CERB_BF16 ? 2 : 4;
  if (a->q_row_stride * es % 16 || a->q_head_stride * es % 16) return CERB_E_ARG;
  if (((uintptr_t)a->q | (uintptr_t)a->k_min | (uintptr_t)a->k_max | (uintptr_t)a->scratch) & 15) return CERB_E_ARG;
  if (s + e + g > a->scratch_bytes || (s + e + g && !a->scratch)) return CERB_E_NOMEM;
  if (a->B == 0) return CERB_OK;
  SelectParams p;
  memset(&p, 0, sizeof(p));
  p.q = a->q;
  p.k_min = a->k_min;
  p.k_max = a->k_max;
  p.page_table = a->page_table;
  p.len = a->len;
  p.sel = a->sel;
  p.n_sel = a->n_sel;
  p.score = (float*)a->scratch;
  p.bound = (float*)((char*)a->scratch + s);
  p.again = (double*)((char*)a->scratch + s + e);
  p.q_row = a->q_row_stride;
  p.q_head = a->q_head_stride;
  p.B = a->B;
  p.H = a->n_heads;
  p.Hk = a->n_kv_heads;
  p.G = a->n_heads / a->n_kv_heads;
  p.max_pages = a->max_pages;
  p.n_pool_pages = a->n_pool_pages;
  p.K = a->max_sel;
  p.n_first = a->n_first;
  p.n_last = a->n_last;
  p.chunks = chunks;
  cudaStream_t st = (cudaStream_t)stream;
  const bool big = a->head_dim == 128, bf = a->dtype == CERB_BF16;
  const unsigned units = (unsigned)(a->B * a->n_kv_heads);
  auto score = bf ? (big ? page_score_bf16_kernel<128> : page_score_bf16_kernel<64>) : (big ? page_score_f32_kernel<128> : page_score_f32_kernel<64>);
  const size_t q_smem = bf ? (size_t)(p.G + 7) / 8 * 8 * (a->head_dim + 8) * sizeof(bf16) : (size_t)p.G * a->head_dim * sizeof(float);
  if (launch_pdl(score, dim3(units * (unsigned)chunks), dim3(SC_WARPS * 32), q_smem, st, p) != cudaSuccess) return CERB_E_CUDA;
  auto kern = bf ? (big ? page_select_kernel<bf16, 128> : page_select_kernel<bf16, 64>) : (big ? page_select_kernel<float, 128> : page_select_kernel<float, 64>);
  static std::atomic<uint64_t> done[4];
  CERB_TRY(allow_smem(kern, done[2 * bf + big], SEL_SMEM_PAGES * (int)sizeof(float)));
  const int held = (int)std::min((long long)a->max_pages, (long long)SEL_SMEM_PAGES);
  return launch_pdl(kern, dim3(units), dim3(SEL_THREADS), (size_t)held * sizeof(float), st, p) == cudaSuccess ? CERB_OK : CERB_E_CUDA;
}

}  // extern "C"
