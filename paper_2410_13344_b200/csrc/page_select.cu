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
//
// Two launches, 24 sequences of up to 32000 tokens (8 KV heads of 128, 117 MB of summaries): scores 22.6 us, 5.2 TB/s; selection 7.2.  One sequence of 131072: 9.2
// and 8.2, of which the fp64 scores of the ten pages near the border are 2; both are rounds of memory latency one after another.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "paged_common.cuh"

namespace cerb {

namespace {

constexpr int SC_WARPS = 4;
constexpr int SEL_KEEP = 8192;              // scores that shared memory keeps: those of caches of up to so many pages
constexpr int SEL_LIST = 512;               // pages near the border that are ranked one against another
// (Page, head) pairs of a unit up to which the selection scores all of its pages itself, in fp64, and no scores are computed ahead of it.  (us with / without, 4 heads, 8 units
// and 256: 32 pages 7.9 / 6.2, 64 pages 7.9 / 9.4; one head: 64 pages 8.4 / 5.7, 128 7.7 / 9.0; 256 units of 8 heads: 16 pages 10.4 / 8.6, 32 pages 10.9 / 14.2.)
constexpr int kScoreAlone = 128;
constexpr int kMaxSelectPages = 1 << 17;    // (a bit mask of them lies in shared memory)

// What is known of the scores of a tile of pages (of those of it that are up for selection).
struct TileScores {
  float bound;                 // of the error of its scores
  float lo, hi;                // smallest and largest score of those that lie in the pool
  int rest;                    // bit 0: scores among them that are not finite; above it the number of pages that lie nowhere
};
constexpr int kTile = 16;      // pages

struct SelectParams {
  const void *q, *k_min, *k_max;
  const int32_t *page_table, *len;
  int32_t *sel, *n_sel;
  float* score;                // [unit][max_pages]
  TileScores* tile;            // [unit][tiles]
  unsigned long long* again;   // [unit][max_pages]: scores of 64 bits as ordered whole numbers
  long long q_row, q_head;     // elements
  int B, H, Hk, G, max_pages, n_pool_pages, K, n_first, n_last, tiles;
  int scored;                  // 0: no scores have been computed, the sequences were to be too short for it
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
__device__ __forceinline__ float larger_size(float a, float b) {         // of |a| and |b|; a NaN if there is one
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
  return r;
}
__device__ __forceinline__ float positive(float a) {                      // the larger of it and zero; a NaN stays one
  float r;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t abs2(uint32_t a) { return a & 0x7fff7fffu; }

// How far a score may be off, relative to S = sum_d |q_d| |k_d|, k_d the one of kmin_d and kmax_d that counts for q_d's sign.
// bf16: q's positive and negative elements are products of their own, Dh / 16 <= 8 steps of the tensor cores each, and a step keeps at least 24 bits of the
// largest of its 17 addends, each of which is at most the product's share of S: 8 x 17 x 2^-23 S, three more roundings and S's own error: under 2^-15.5 S.
// fp32: chains of at most Dh / 32 + 5 roundings (one of q_d's two products is a zero, which is added exactly): under 2^-19 S.  Its S is one for all heads, of the largest |q_d| among
// them and the larger of |kmin_d| and |kmax_d|.
// A sum of so small numbers that its products or steps underflow is off by less than 2^-126 for each of them besides: kUnderflow.
template <typename T> __device__ __forceinline__ float error_factor();
template <> __device__ __forceinline__ float error_factor<bf16>() { return 2.1579186e-5f; }
template <> __device__ __forceinline__ float error_factor<float>() { return 1.0f / 524288; }
constexpr float kUnderflow = 2.4074124e-35f;                             // 2^-115, 2048 of them

// Leaves what a warp's lanes know of a tile.
__device__ __forceinline__ void leave_tile(TileScores* to, float bound, float lo, float hi, bool odd, int nowhere) {
#pragma unroll
  for (int w = 1; w < 32; w <<= 1) {
    bound = fmaxf(bound, __shfl_xor_sync(0xffffffffu, bound, w));
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, w));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, w));
  }
  odd = __any_sync(0xffffffffu, odd);
  nowhere = __reduce_add_sync(0xffffffffu, nowhere);
  if ((threadIdx.x & 31) == 0) *reinterpret_cast<float4*>(to) = make_float4(bound, lo, hi, __int_as_float(2 * nowhere + odd));
}

// A warp's way through its share of the tiles of all units whose pages have to be selected from.
struct TileWalk {
  int b, kvh, tile, N, tiles;  // of the present one: sequence, KV head, tile, the sequence's pages and tiles
  long long left;              // with the present one
};
__device__ __forceinline__ int tiles_of(const SelectParams& p, int b) {
  const int N = pages_held(p, b);
  return N > p.K ? (N + kTile - 1) / kTile : 0;
}
__device__ __forceinline__ TileWalk walk_tiles(const SelectParams& p) {
  const Share s = share_of(p.B, [&](int b) { return (long long)tiles_of(p, b) * p.Hk; }, blockIdx.x * SC_WARPS + (threadIdx.x >> 5), gridDim.x * SC_WARPS, 1, 1);
  TileWalk w;
  w.left = s.end - s.begin;
  w.b = s.b;
  if (w.left <= 0) return w;
  w.N = pages_held(p, w.b);
  w.tiles = tiles_of(p, w.b);
  w.kvh = (int)((unsigned)s.off / (unsigned)w.tiles);                    // (less than 2^31: a sequence has 2^13 tiles at most, and 2^16 KV heads)
  w.tile = (int)((unsigned)s.off - (unsigned)w.kvh * w.tiles);
  return w;
}
__device__ __forceinline__ void next_tile(const SelectParams& p, TileWalk& w) {
  if (--w.left <= 0 || ++w.tile < w.tiles) return;
  w.tile = 0;
  if (++w.kvh < p.Hk) return;
  w.kvh = 0;
  do w.tiles = tiles_of(p, ++w.b);
  while (w.tiles == 0);
  w.N = pages_held(p, w.b);
}

// bf16 scores: 16 pages on the rows of a warp MMA, eight heads on its columns, kmax and kmin straight from global memory in the order in which the lanes
// load them, the next 16 pages' on their way.  S is a product like the scores, of absolute values.
template <int DH>
__global__ void __launch_bounds__(SC_WARPS * 32, 3) page_score_bf16_kernel(const SelectParams p) {
  constexpr int KC = DH / 32;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  griddep_wait();
  TileWalk now = walk_tiles(p);
  struct Pages {
    int at[2];
  };
  auto find = [&](const TileWalk& w) {
    Pages x;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int page = w.tile * kTile + g + 8 * e;
      x.at[e] = w.left > 0 && page < w.N ? page_at(p, w.b, page) : -1;
    }
    return x;
  };
  auto load = [&](uint4 (&x)[2][KC], const void* from, const TileWalk& w, const Pages& pages) {
    const bf16* src = reinterpret_cast<const bf16*>(from) + (size_t)w.kvh * DH + 8 * t;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        x[e][j] = make_uint4(0, 0, 0, 0);
        if (pages.at[e] >= 0) x[e][j] = ld16(src + (size_t)pages.at[e] * p.Hk * DH + 32 * j);
      }
  };
  uint4 hi[2][KC], lo[2][KC], q[KC];
  TileWalk then = now;
  if (then.left > 0) next_tile(p, then);
  Pages pages = find(now), pages_then = find(then);
  load(hi, p.k_max, now, pages);
  load(lo, p.k_min, now, pages);
  const int tiles = (p.G + 7) / 8;
  int have = -1;                                                         // the (sequence, KV head) of the queries that are in q, where they all fit
  while (now.left > 0) {
    TileWalk after = then;
    if (after.left > 0) next_tile(p, after);
    const Pages pages_after = find(after);
    const int unit = now.b * p.Hk + now.kvh;
    float best[2] = {-INFINITY, -INFINITY}, bound = 0.f;
    bool nan[2] = {false, false};
    for (int n = 0; n < tiles; ++n) {
      if (tiles > 1 || unit != have) {
        have = unit;
        const bf16* src = reinterpret_cast<const bf16*>(p.q) + (size_t)now.b * p.q_row + (size_t)(now.kvh * p.G + 8 * n + g) * p.q_head + 8 * t;
#pragma unroll
        for (int j = 0; j < KC; ++j) q[j] = 8 * n + g < p.G ? *reinterpret_cast<const uint4*>(src + 32 * j) : make_uint4(0, 0, 0, 0);
      }
      float sh[4] = {0.f, 0.f, 0.f, 0.f}, sl[4] = {0.f, 0.f, 0.f, 0.f}, bh[4] = {0.f, 0.f, 0.f, 0.f}, bl[4] = {0.f, 0.f, 0.f, 0.f};
      auto multiply = [&](const uint4 (&x)[2][KC], bool up, float (&s)[4], float (&a)[4]) {
#pragma unroll
        for (int j = 0; j < KC; ++j) {
          const uint32_t qw[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
          const uint32_t x0[4] = {x[0][j].x, x[0][j].y, x[0][j].z, x[0][j].w}, x1[4] = {x[1][j].x, x[1][j].y, x[1][j].z, x[1][j].w};
#pragma unroll
          for (int w = 0; w < 4; w += 2) {
            const uint32_t q0 = up ? max2(qw[w], 0u) : min2(qw[w], 0u), q1 = up ? max2(qw[w + 1], 0u) : min2(qw[w + 1], 0u);
            mma_16816(s, x0[w], x1[w], x0[w + 1], x1[w + 1], q0, q1);
            mma_16816(a, abs2(x0[w]), abs2(x1[w]), abs2(x0[w + 1]), abs2(x1[w + 1]), abs2(q0), abs2(q1));
          }
        }
      };
      multiply(hi, true, sh, bh);
      if (n == tiles - 1) load(hi, p.k_max, then, pages_then);
      multiply(lo, false, sl, bl);
      if (n == tiles - 1) load(lo, p.k_min, then, pages_then);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (8 * n + 2 * t + (e & 1) >= p.G) continue;
        const float s = sh[e] + sl[e], a = bh[e] + bl[e];
        nan[e >> 1] |= s != s;
        best[e >> 1] = fmaxf(best[e >> 1], s);
        if (pages.at[e >> 1] >= 0) bound = a == a ? fmaxf(bound, a) : INFINITY;
      }
    }
    float least = INFINITY, most = -INFINITY;
    bool odd = false;
    int nowhere = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float s = nan[e] ? NAN : best[e];
#pragma unroll
      for (int w = 1; w < 4; w <<= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, s, w);
        s = s != s || other != other ? NAN : fmaxf(s, other);
      }
      const int page = now.tile * kTile + g + 8 * e;
      if (pages.at[e] < 0) s = -INFINITY;                                // (a page that lies nowhere: below every other)
      if (page < now.N) {
        if (t == 0) p.score[(size_t)unit * p.max_pages + page] = s;
        if (page >= p.n_first && page < now.N - p.n_last) {
          if (pages.at[e] < 0) {
            nowhere += t == 0;
          } else {
            odd |= !(fabsf(s) < INFINITY);
            least = fminf(least, s);
            most = fmaxf(most, s);
          }
        }
      }
    }
    leave_tile(p.tile + (size_t)unit * p.tiles + now.tile, bound * error_factor<bf16>() + kUnderflow, least, most, odd, nowhere);
    now = then;
    pages = pages_then;
    then = after;
    pages_then = pages_after;
  }
}

// fp32 scores: half a tile to a warp at a time, DH / 32 elements to a lane, FMA on pairs; the scores of a head are eight sums over the lanes, and so is S.
// (With S for every head by itself, and a choice between kmin and kmax before the product: scores and selection of 8 units of 5021 pages, 16 heads of 128, 46.9 us instead of 32.2.)
template <int DH>
__global__ void __launch_bounds__(SC_WARPS * 32, 4) page_score_f32_kernel(const SelectParams p) {
  constexpr int E = DH / 32, PAGES = 8;
  struct alignas(4 * E) Elems {
    float x[E];
  };
  struct alignas(4 * E) Pairs {
    f32x2 x[E / 2];
  };
  const int lane = threadIdx.x & 31;
  griddep_wait();
  float most_q[E];                                                       // of the heads of `have`
  int have = -1;
  for (TileWalk now = walk_tiles(p); now.left > 0; next_tile(p, now)) {
    const int unit = now.b * p.Hk + now.kvh;
    const Pairs* src_hi = reinterpret_cast<const Pairs*>(p.k_max) + (size_t)now.kvh * 32 + lane;
    const Pairs* src_lo = reinterpret_cast<const Pairs*>(p.k_min) + (size_t)now.kvh * 32 + lane;
    const float* src_q = reinterpret_cast<const float*>(p.q) + (size_t)now.b * p.q_row + (size_t)now.kvh * p.G * p.q_head + lane * E;
    const int of_tile = lane < kTile && now.tile * kTile + lane < now.N ? page_at(p, now.b, now.tile * kTile + lane) : -1;
    if (unit != have) {
      have = unit;
#pragma unroll
      for (int e = 0; e < E; ++e) most_q[e] = 0.f;
#pragma unroll 4
      for (int h = 0; h < p.G; ++h) {
        const Elems x = *reinterpret_cast<const Elems*>(src_q + h * p.q_head);
#pragma unroll
        for (int e = 0; e < E; ++e) most_q[e] = larger_size(most_q[e], x.x[e]);
      }
    }
    float bound = 0.f, least = INFINITY, most = -INFINITY;
    bool odd = false;
    int nowhere = 0;
#pragma unroll 1
    for (int half = 0; half < kTile / PAGES; ++half) {
      Pairs hi[PAGES], lo[PAGES];
#pragma unroll
      for (int j = 0; j < PAGES; ++j) {
        const int at = __shfl_sync(0xffffffffu, of_tile, half * PAGES + j);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) hi[j].x[e] = lo[j].x[e] = 0;
        if (at >= 0) {
          hi[j] = src_hi[(size_t)at * p.Hk * 32];
          lo[j] = src_lo[(size_t)at * p.Hk * 32];
        }
      }
      float s[PAGES];
#pragma unroll
      for (int j = 0; j < PAGES; ++j) {
        s[j] = 0.f;
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const float2 h = parts_of(hi[j].x[e]), l = parts_of(lo[j].x[e]);
          s[j] = fmaf(most_q[2 * e], larger_size(h.x, l.x), s[j]);
          s[j] = fmaf(most_q[2 * e + 1], larger_size(h.y, l.y), s[j]);
        }
      }
      halve_sums(s, lane);                                               // lane: of page lane / 4
      const float far = s[0] == s[0] ? s[0] : INFINITY;
      float best = -INFINITY;
      bool nan = false;
#pragma unroll 2
      for (int h = 0; h < p.G; ++h) {
        const Elems x = *reinterpret_cast<const Elems*>(src_q + h * p.q_head);
        f32x2 up[E / 2], down[E / 2];
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          up[e / 2] = pair_of(positive(x.x[e]), positive(x.x[e + 1]));
          down[e / 2] = pair_of(-positive(-x.x[e]), -positive(-x.x[e + 1]));
        }
#pragma unroll
        for (int j = 0; j < PAGES; ++j) {
          f32x2 sum = mul2(up[0], hi[j].x[0]);
          sum = fma2(down[0], lo[j].x[0], sum);
#pragma unroll
          for (int e = 1; e < E / 2; ++e) {
            sum = fma2(up[e], hi[j].x[e], sum);
            sum = fma2(down[e], lo[j].x[e], sum);
          }
          const float2 y = parts_of(sum);
          s[j] = y.x + y.y;
        }
        halve_sums(s, lane);
        nan |= s[0] != s[0];
        best = fmaxf(best, s[0]);
      }
      const int i = half * PAGES + lane / 4, page = now.tile * kTile + i, at = __shfl_sync(0xffffffffu, of_tile, i);
      if (at >= 0) bound = fmaxf(bound, far);
      if (page < now.N) {
        const float x = at < 0 ? -INFINITY : nan ? NAN : best;
        if (lane % 4 == 0) p.score[(size_t)unit * p.max_pages + page] = x;
        if (page >= p.n_first && page < now.N - p.n_last) {
          if (at < 0) {
            nowhere += lane % 4 == 0;
          } else {
            odd |= !(fabsf(x) < INFINITY);
            least = fminf(least, x);
            most = fmaxf(most, x);
          }
        }
      }
    }
    leave_tile(p.tile + (size_t)unit * p.tiles + now.tile, bound * error_factor<float>() + kUnderflow, least, most, odd, nowhere);
  }
}

// A page's score for one head in fp64, by eight lanes (all 32 of the warp call).  `at`: where the page lies, -1: nowhere.
template <typename T> __device__ __forceinline__ float wide(T x);
template <> __device__ __forceinline__ float wide<float>(float x) { return x; }
template <> __device__ __forceinline__ float wide<bf16>(bf16 x) { return __bfloat162float(x); }
template <typename T, int DH>
__device__ __forceinline__ double score_again(const SelectParams& p, int b, int kvh, int at, int head, int lane) {
  constexpr int E = 16 / sizeof(T);                                      // elements of a load
  struct alignas(16) Elems {
    T x[E];
  };
  constexpr int J = DH / (8 * E);
  const size_t from = ((size_t)max(at, 0) * p.Hk + kvh) * DH + lane % 8 * E;
  const T* hi = reinterpret_cast<const T*>(p.k_max) + from;
  const T* lo = reinterpret_cast<const T*>(p.k_min) + from;
  const T* q = reinterpret_cast<const T*>(p.q) + (size_t)b * p.q_row + (size_t)(kvh * p.G + head) * p.q_head + lane % 8 * E;
  Elems h[J], l[J], x[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    h[j] = *reinterpret_cast<const Elems*>(hi + j * 8 * E);
    l[j] = *reinterpret_cast<const Elems*>(lo + j * 8 * E);
    x[j] = *reinterpret_cast<const Elems*>(q + j * 8 * E);
  }
  double sum[2] = {0.0, 0.0};
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      // the larger product is the one with kmax where q is positive, with kmin where it is negative; where q is zero, and where one of them is not a
      // number, the one that makes the sum what the definition makes it
      const float y = wide<T>(x[j].x[e]), c = wide<T>(h[j].x[e]), a = wide<T>(l[j].x[e]);
      float k = y > 0.f || (y == 0.f && fabsf(c) >= fabsf(a)) ? c : a;
      if (c != c) k = c;
      if (a != a) k = a;
      sum[e & 1] = fma((double)y, (double)k, sum[e & 1]);
    }
  double s = sum[0] + sum[1];
#pragma unroll
  for (int w = 4; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
  return at < 0 ? -INFINITY : s;
}

// Order-preserving images of floats and doubles.
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i >= 0 ? i : i ^ 0x7fffffff;
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i >= 0 ? i : i ^ 0x7fffffff); }
__device__ __forceinline__ unsigned long long ordered(double x) {
  if (x == 0.0) x = 0.0;                                                 // (one zero)
  if (x != x) x = INFINITY;                                              // (what is not a number ranks first)
  const unsigned long long i = (unsigned long long)__double_as_longlong(x);
  return i >> 63 ? ~i : i | 0x8000000000000000ull;
}

template <int SEL_THREADS>
__device__ __forceinline__ int block_sum(int v, int* red) {
  constexpr int WARPS = SEL_THREADS / 32;
  const int lane = threadIdx.x & 31;
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if (lane == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, lane < WARPS ? red[lane] : 0);
}
template <int SEL_THREADS>
__device__ __forceinline__ int block_scan(int v, int* red, int& total) {     // exclusive
  constexpr int WARPS = SEL_THREADS / 32;
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
  int w = lane < WARPS ? red[lane] : 0;
#pragma unroll
  for (int o = 1; o < WARPS; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += u;
  }
  total = __shfl_sync(0xffffffffu, w, WARPS - 1);
  const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
  return s - v + (warp ? before : 0);
}

// One CTA per (sequence, KV head).  The border is closed in on by histograms between the smallest and the largest score (a bin is a range of values; a score's
// bin is a monotonic function of it), each level in the range of the bin that holds the border, until few pages are left in it; those, and
// what lies within 2 E of them, are ranked in fp64.  Scores of up to SEL_KEEP pages stay in shared memory, those of more are read again at every pass.
// With a CTA to an SM, each of its instructions executed a few times, much of the time is that of fetching them: the loops stay rolled.  (Unrolled, with
// the scores in registers, the histogram of 2000 pages took as long as that of 8192, 3 us.)
template <typename T, int DH, int SEL_THREADS>
__global__ void __launch_bounds__(SEL_THREADS, 1024 / SEL_THREADS) page_select_kernel(const SelectParams p) {
  constexpr int SEL_BINS = SEL_THREADS;
  __shared__ int red[32], hist[SEL_BINS];
  __shared__ int list[SEL_LIST], list_at[SEL_LIST];
  __shared__ unsigned long long again[SEL_LIST];
  __shared__ int s_lo, s_hi, s_n, s_bin, s_above, s_bound, s_odd, s_nowhere;
  extern __shared__ unsigned taken[];                                    // a bit for each page of the table's row, then the scores that are kept
  float* kept = reinterpret_cast<float*>(taken + (p.max_pages + 31) / 32);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, kvh = unit % p.Hk, b = unit / p.Hk;
  if (tid == 0) {
    s_lo = ordered(INFINITY);
    s_hi = ordered(-INFINITY);
    s_n = s_bound = s_odd = s_nowhere = 0;
  }
  hist[tid] = 0;
  griddep_wait();
  griddep_launch();
  // what does not need the length is on its way before it: the scores (of the whole table's row, whatever lies behind the last) and what is known of them
  const float* score = p.score + (size_t)unit * p.max_pages;
  for (int i = tid; p.scored && i < min(p.max_pages, SEL_KEEP); i += SEL_THREADS)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(kept + i)), "l"(score + i) : "memory");
  const float4* of_tile = reinterpret_cast<const float4*>(p.tile + (size_t)unit * p.tiles);
  float4 known = make_float4(0.f, INFINITY, -INFINITY, 0.f);
  if (p.scored && tid < p.tiles) known = of_tile[tid];
  const int N = pages_held(p, b), n = min(N, p.K);
  int32_t* sel = p.sel + (size_t)unit * p.K;
  if (kvh == 0 && tid == 0) p.n_sel[b] = n;
  for (int i = n + tid; i < p.K; i += SEL_THREADS) sel[i] = -1;
  if (N <= p.K) {
    for (int i = tid; i < N; i += SEL_THREADS) sel[i] = i;
    asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  const int first = p.n_first, last = N - p.n_last;                      // pages first .. last - 1 are up for selection
  const int want = p.K - first - p.n_last;                               // (K >= n_first + n_last, and N > K)
  const bool keep = N <= SEL_KEEP;                                       // (without scores: whatever lies there, which nothing is decided by)
  // f(page, score) for this thread's pages
  auto each = [&](auto f) {
    if (keep) {
#pragma unroll 1
      for (int i = first + tid; i < last; i += 4 * SEL_THREADS) {
        float s[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = i + j * SEL_THREADS < last ? kept[i + j * SEL_THREADS] : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (i + j * SEL_THREADS < last) f(i + j * SEL_THREADS, s[j]);
      }
    } else {
#pragma unroll 1
      for (int i = first + tid; i < last; i += SEL_THREADS) f(i, score[i]);
    }
  };
  const int words = (N + 31) / 32;
  auto below = [](int pages, int word) { return pages >= word * 32 + 32 ? 0xffffffffu : pages <= word * 32 ? 0u : (1u << (pages - word * 32)) - 1; };
  for (int i = tid; i < words; i += SEL_THREADS) taken[i] = below(first, i) | (below(N, i) & ~below(last, i));    // the ones that are always taken
  __syncthreads();
  if (p.scored) {
    const int tiles = (N + kTile - 1) / kTile;
    if (tid >= tiles) known = make_float4(0.f, INFINITY, -INFINITY, 0.f);
    bool odd = __float_as_int(known.w) & 1;
    int nowhere = __float_as_int(known.w) >> 1;
    for (int i = tid + SEL_THREADS; i < tiles; i += SEL_THREADS) {
      const float4 k = of_tile[i];
      known.x = fmaxf(known.x, k.x);
      known.y = fminf(known.y, k.y);
      known.z = fmaxf(known.z, k.z);
      odd |= __float_as_int(k.w) & 1;
      nowhere += __float_as_int(k.w) >> 1;
    }
    if (tid / 32 * 32 < tiles) {
      const int lw = __reduce_min_sync(0xffffffffu, ordered(known.y)), hw = __reduce_max_sync(0xffffffffu, ordered(known.z));
      const int e = __reduce_max_sync(0xffffffffu, __float_as_int(known.x));   // (not negative, not a NaN)
      odd = __any_sync(0xffffffffu, odd);
      nowhere = __reduce_add_sync(0xffffffffu, nowhere);
      if (lane == 0) {
        if (nowhere) atomicAdd(&s_nowhere, nowhere);
        atomicMin(&s_lo, lw);
        atomicMax(&s_hi, hw);
        atomicMax(&s_bound, e);
        if (odd) s_odd = 1;
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  const float E = __int_as_float(s_bound);
  float lo = from_ordered(s_lo), hi = from_ordered(s_hi);
  const bool all_again = !p.scored || s_odd || !(E < INFINITY);          // scores that are not finite decide nothing
  int above = 0;                                                         // pages above hi
  float t_lo = -INFINITY, t_hi = INFINITY;
  if (!all_again && last - first - s_nowhere <= want) {
    t_hi = -INFINITY;                                                    // all pages that lie in the pool, and the first ones of the others
  } else if (!all_again && want > 0) {
#pragma unroll 1
    for (int level = 0; level < 8; ++level) {
      const float range = hi - lo, inv = (float)SEL_BINS / range;
      if (!(hi > lo) || !(range < INFINITY) || !(inv < INFINITY)) break;    // (finite scores further apart than fp32 reaches: all of them are near)
      auto bin_of = [&](float s) { return min(SEL_BINS - 1, max(0, (int)((s - lo) * inv))); };
      if (level) {
        __syncthreads();
        hist[tid] = 0;
        __syncthreads();
      }
      each([&](int, float s) {
        if (s >= lo && s <= hi) atomicAdd(&hist[bin_of(s)], 1);
      });
      __syncthreads();
      // the bin with the want-th best: thread i looks at the i-th bin from above
      const int mine = hist[SEL_BINS - 1 - tid];
      int total;
      const int before = above + block_scan<SEL_THREADS>(mine, red, total);
      if (before < want && before + mine >= want) { s_bin = SEL_BINS - 1 - tid; s_above = before; s_lo = ordered(INFINITY); s_hi = ordered(-INFINITY); }
      __syncthreads();
      const int bin = s_bin, count = hist[bin];
      above = s_above;
      if (count <= 32) {
        // the bin's edges, and more than what rounding can have moved a score across them
        const float slack = 4e-7f * (fabsf(lo) + fabsf(hi)), from = lo;
        lo = from + (float)bin / inv - slack;
        hi = from + (float)(bin + 1) / inv + slack;
        break;
      }
      float l = INFINITY, h = -INFINITY;
      each([&](int, float s) {
        if (s >= lo && s <= hi && bin_of(s) == bin) { l = fminf(l, s); h = fmaxf(h, s); }
      });
      if (__any_sync(0xffffffffu, l <= h)) {
        const int lw = __reduce_min_sync(0xffffffffu, ordered(l)), hw = __reduce_max_sync(0xffffffffu, ordered(h));
        if (lane == 0) { atomicMin(&s_lo, lw); atomicMax(&s_hi, hw); }
      }
      __syncthreads();
      lo = from_ordered(s_lo);
      hi = from_ordered(s_hi);
      if (hi - lo <= E) break;
    }
    t_lo = lo - 2.1f * E;
    t_hi = hi + 2.1f * E;
  }
  // sure ones and those near the border
  int sure = 0;
  if (want > 0)
    each([&](int i, float s) {
      if (!all_again && s > t_hi) {
        atomicOr(&taken[i >> 5], 1u << (i & 31));
        ++sure;
      } else if (all_again || s >= t_lo) {
        const int at = atomicAdd(&s_n, 1);
        if (at < SEL_LIST) { list[at] = i; list_at[at] = page_at(p, b, i); again[at] = 0; }
      }
    });
  sure = block_sum<SEL_THREADS>(sure, red);
  const int near = s_n, rest = want - sure;
  if (near <= SEL_LIST) {
    if (near > rest) {
#pragma unroll 1
      for (int i0 = warp * 4; i0 < near * p.G; i0 += SEL_THREADS / 8) {
        const int i = i0 + lane / 8, w = min(i, near * p.G - 1);
        const double s = score_again<T, DH>(p, b, kvh, list_at[w / p.G], w % p.G, lane);
        if (lane % 8 == 0 && i == w) atomicMax(&again[w / p.G], ordered(s));
      }
      __syncthreads();
    }
    // a page's rank among them, by a warp
#pragma unroll 1
    for (int i = warp; i < near; i += SEL_THREADS / 32) {
      int rank = 0;
      if (near > rest) {
        const unsigned long long mine = again[i];
        const int page = list[i];
        for (int j = lane; j - lane < near; j += 32) {
          const unsigned long long other = j < near ? again[j] : 0;
          rank += __popc(__ballot_sync(0xffffffffu, other > mine || (other == mine && j < near && list[j] < page)));
        }
      }
      if (lane == 0 && rank < rest) atomicOr(&taken[list[i] >> 5], 1u << (list[i] & 31));
    }
  } else {
    // many near the border (a cache of equal keys, scores that are not finite): all of them in fp64, the border by bisection of the ordered values
    unsigned long long* far = p.again + (size_t)unit * p.max_pages;
    auto is_near = [&](int i) { return all_again || (score[i] >= t_lo && score[i] <= t_hi); };
#pragma unroll 1
    for (int i0 = first + warp * 4; i0 < last; i0 += SEL_THREADS / 8) {
      const int i = min(i0 + lane / 8, last - 1), at = page_at(p, b, i);
      unsigned long long best = 0;
#pragma unroll 1
      for (int h = 0; h < p.G; ++h) best = max(best, ordered(score_again<T, DH>(p, b, kvh, at, h, lane)));
      if (lane % 8 == 0) far[i] = best;
    }
    __syncthreads();
    unsigned long long v = 0;                                            // the largest that `rest` or more are not below
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long c = v | 1ull << bit;
      int cnt = 0;
#pragma unroll 4
      for (int i = first + tid; i < last; i += SEL_THREADS) cnt += is_near(i) && far[i] >= c;
      if (block_sum<SEL_THREADS>(cnt, red) >= rest) v = c;
    }
    int over = 0;
    for (int i = first + tid; i < last; i += SEL_THREADS)
      if (is_near(i) && far[i] > v) {
        atomicOr(&taken[i >> 5], 1u << (i & 31));
        ++over;
      }
    int ties = rest - block_sum<SEL_THREADS>(over, red);
    for (int i0 = first; i0 < last && ties > 0; i0 += SEL_THREADS) {
      const int i = i0 + tid;
      const int tie = i < last && is_near(i) && far[i] == v;
      int total;
      const int before = block_scan<SEL_THREADS>(tie, red, total);
      if (tie && before < ties) atomicOr(&taken[i >> 5], 1u << (i & 31));
      ties -= total;
    }
  }
  __syncthreads();
  int written = 0;
  for (int w0 = 0; w0 < words; w0 += SEL_THREADS) {
    unsigned m = w0 + tid < words ? taken[w0 + tid] : 0;
    int total, at = written + block_scan<SEL_THREADS>(__popc(m), red, total);
    for (; m; m &= m - 1) sel[at++] = (w0 + tid) * 32 + __ffs(m) - 1;
    written += total;
  }
}

struct SelectPlan {
  int ctas, tiles;
  size_t score_bytes, tile_bytes, again_bytes;
};
int plan_select(int dtype, int B, int H, int Hk, int head_dim, int max_pages, int max_len, SelectPlan* g) {
  if (dtype != CERB_F32 && dtype != CERB_BF16) return CERB_E_ARG;
  if (B < 0 || H < 1 || Hk < 1 || H % Hk || (head_dim != 64 && head_dim != 128) || max_pages < 1 || max_pages > kMaxSelectPages) return CERB_E_SHAPE;
  if (H / Hk > 64 || Hk > 0xffff || (long long)B * Hk > 0x7fffffll) return CERB_E_SHAPE;
  const long long units = (long long)B * Hk;
  g->tiles = (max_pages + kTile - 1) / kTile;
  // as many CTAs as run at once, of no less than a tile to a warp
  const int held = (int)std::min(((long long)max_len + CERB_PAGE - 1) / CERB_PAGE, (long long)max_pages);
  const long long most = (units * ((held + kTile - 1) / kTile) + SC_WARPS - 1) / SC_WARPS;
  g->ctas = (int)std::max(1ll, std::min(most, 148ll * (dtype == CERB_BF16 ? 3 : 4)));
  g->score_bytes = ((size_t)units * max_pages * sizeof(float) + 255) & ~(size_t)255;
  g->tile_bytes = ((size_t)units * g->tiles * sizeof(TileScores) + 255) & ~(size_t)255;
  g->again_bytes = (size_t)units * max_pages * sizeof(unsigned long long);
  return CERB_OK;
}

template <typename T, int DH, int THREADS>
int launch_select(const SelectParams& p, unsigned units, size_t smem, cudaStream_t st) {
  auto kern = page_select_kernel<T, DH, THREADS>;
  static std::atomic<uint64_t> done{0};
  CERB_TRY(allow_smem(kern, done, kMaxSelectPages / 8 + SEL_KEEP * (int)sizeof(float)));
  return launch_pdl(kern, dim3(units), dim3(THREADS), smem, st, p) == cudaSuccess ? CERB_OK : CERB_E_CUDA;
}

}  // namespace

}  // namespace cerb

using namespace cerb;

extern "C" {

int cerb_page_select_scratch_bytes(int32_t dtype, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_pages, int32_t max_len,
                                   size_t* bytes_out) {
  if (!bytes_out || max_len < 1) return CERB_E_ARG;
  SelectPlan g;
  CERB_TRY(plan_select(dtype, B, n_heads, n_kv_heads, head_dim, max_pages, max_len, &g));
  *bytes_out = g.score_bytes + g.tile_bytes + g.again_bytes;
  return CERB_OK;
}

int cerb_page_select(const cerb_page_select_args* a, void* stream) {
  if (!a || (a->B > 0 && (!a->q || !a->k_min || !a->k_max || !a->page_table || !a->len || !a->sel || !a->n_sel))) return CERB_E_ARG;
  if (a->n_pool_pages < 1 || a->max_len < 1 || a->n_first < 0 || a->n_last < 0 || a->max_sel < 1) return CERB_E_ARG;
  if ((long long)a->n_first + a->n_last > a->max_sel || a->max_sel > kMaxList) return CERB_E_SHAPE;
  SelectPlan g;
  CERB_TRY(plan_select(a->dtype, a->B, a->n_heads, a->n_kv_heads, a->head_dim, a->max_pages, a->max_len, &g));
  const int es = a->dtype == CERB_BF16 ? 2 : 4;
  if (a->q_row_stride * es % 16 || a->q_head_stride * es % 16) return CERB_E_ARG;
  if (((uintptr_t)a->q | (uintptr_t)a->k_min | (uintptr_t)a->k_max | (uintptr_t)a->scratch) & 15) return CERB_E_ARG;
  const size_t need = g.score_bytes + g.tile_bytes + g.again_bytes;
  if (need > a->scratch_bytes || (need && !a->scratch)) return CERB_E_NOMEM;
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
  p.tile = (TileScores*)((char*)a->scratch + g.score_bytes);
  p.again = (unsigned long long*)((char*)a->scratch + g.score_bytes + g.tile_bytes);
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
  p.tiles = g.tiles;
  cudaStream_t st = (cudaStream_t)stream;
  const bool big = a->head_dim == 128, bf = a->dtype == CERB_BF16;
  const unsigned units = (unsigned)(a->B * a->n_kv_heads);
  auto score = bf ? (big ? page_score_bf16_kernel<128> : page_score_bf16_kernel<64>) : (big ? page_score_f32_kernel<128> : page_score_f32_kernel<64>);
  // (a sequence that is longer than the caller said has all of its pages scored in fp64)
  const long long held = ((long long)a->max_len + CERB_PAGE - 1) / CERB_PAGE;
  p.scored = held > a->max_sel && held * p.G > kScoreAlone;
  if (p.scored && launch_pdl(score, dim3((unsigned)g.ctas), dim3(SC_WARPS * 32), 0, st, p) != cudaSuccess) return CERB_E_CUDA;
  const size_t smem = ((size_t)a->max_pages + 31) / 32 * sizeof(unsigned) + std::min(a->max_pages, SEL_KEEP) * sizeof(float);
  // (twice the threads while every unit has an SM to itself)
  if (units <= 148)
    return bf ? (big ? launch_select<bf16, 128, 1024>(p, units, smem, st) : launch_select<bf16, 64, 1024>(p, units, smem, st))
              : (big ? launch_select<float, 128, 1024>(p, units, smem, st) : launch_select<float, 64, 1024>(p, units, smem, st));
  return bf ? (big ? launch_select<bf16, 128, 512>(p, units, smem, st) : launch_select<bf16, 64, 512>(p, units, smem, st))
            : (big ? launch_select<float, 128, 512>(p, units, smem, st) : launch_select<float, 64, 512>(p, units, smem, st));
}

}  // extern "C"
