// Attention of one new token per sequence over a paged cache whose KV heads are shared by groups of query heads, all of it or the pages of a list.
//
//   out[b][h] = sum_s softmax_s(scale q[b][h] . k[s]) v[s],  lse = ln sum_s exp(scale q . k[s]),
//   s over the slots [max(0, len - window), len), with a list over those of them that lie in its pages.
//
// Bound by HBM: every key and value once, for all query heads of a unit (a KV head's group of them, or eight or sixteen of a larger one).  A warp takes a page of 16
// keys at a time, alone, from global memory straight into the fragments of warp MMAs: no shared memory, no barriers until the end.  (Through a ring in shared memory, filled by
// asynchronous copies: 64 sequences of up to 8192 tokens 221 us instead of 196, a selection of 24 x 128 pages 73 instead of 66; more instructions a page, and less L1 for the loads of
// what runs next to it.)  The sums run as one online softmax per warp.  Who meets, in three forms:
//   - a warp per unit, many short sequences: nobody;
//   - a cluster per unit: the warps of a CTA in shared memory, its CTAs in each other's;
//   - shares, long caches: all units' pages one after another in equal parts, one per CTA of a single wave; units that were cut are joined by a second kernel.
// 64 sequences of up to 8192 tokens (64 heads on 8, heads of 128, 1257 MB) 187 us and 4 for the join: 6.7 TB/s in the main kernel, the rate of a copy; CTAs of equal shares
// end between 172 and 187.  One sequence of 1000 tokens (32 heads on 8) 5.3 us a pass: 2.0 to the first keys' arrival, 0.4 for their products, the rest the meeting and the launch.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "paged_common.cuh"
#include "tc_common.cuh"

namespace cerb {

namespace {

constexpr int PA_WARPS = 4;
constexpr int PA_CLUSTER = 16;        // CTAs of a cluster at most
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PagedParams {
  const void *q, *k_pool, *v_pool;
  const int32_t *page_table, *len, *sel, *n_sel;
  void* out;
  float* lse;
  float *part_o, *part_ml;        // [2 * CTAs][heads of a unit][Dh], [..][2]
  int4* meta;                     // [joins]: unit, first part, number of parts (1 or less: nothing to join)
  long long q_row, q_head;        // elements
  int B, H, Hk, G, units_h;       // units_h: units per KV head (groups of more heads than a unit takes)
  int max_pages, n_pool_pages, max_sel, window;
  int min_share, by_unit;         // by_unit: a join per unit, else one per CTA
  int together;                   // CTAs of a cluster
  float scale_log2;
};

// What a sequence's slots are: [lo, hi), and the items (pages or list entries) that are looked at.
struct Span {
  int lo, hi, first, items;
};
__device__ __forceinline__ Span span_of(const PagedParams& p, int b) {
  Span s;
  s.hi = min(max(p.len[b], 0), p.max_pages * CERB_PAGE);
  s.lo = p.window > 0 ? max(0, s.hi - p.window) : 0;
  s.first = p.sel ? 0 : s.lo / CERB_PAGE;
  s.items = p.sel ? min(max(p.n_sel[b], 0), p.max_sel) : (s.hi + CERB_PAGE - 1) / CERB_PAGE - s.first;
  if (s.hi == 0) s.items = 0;
  return s;
}

// The page of an item: its number among the sequence's, and where it lies (-1: nowhere in the pool).  Needs the sequence's length only for `first`: what lies
// behind it, or behind the list, is for the caller to leave out.
struct PageRef {
  int page, at;
};
__device__ __forceinline__ PageRef page_ref(const PagedParams& p, int first, int b, int kvh, int item) {
  PageRef r{-1, -1};
  if (p.sel) {
    if (item < p.max_sel) r.page = p.sel[((size_t)b * p.Hk + kvh) * p.max_sel + item];
  } else {
    r.page = first + item;
  }
  if (r.page < 0 || r.page >= p.max_pages) return r;
  const int at = p.page_table[(size_t)b * p.max_pages + r.page];
  if (at < p.n_pool_pages) r.at = at;
  return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The running maxima, sums and unnormalised outputs of a CTA's warps.
template <int DH, int HEADS>
struct alignas(16) Sums {                                                // (written and sent in pieces of 8 bytes)
  float o[PA_WARPS][HEADS][DH], m[PA_WARPS][HEADS], l[PA_WARPS][HEADS];
};
// Four columns of a head from d on, with its maximum and sum.
template <int DH, int HEADS>
__device__ __forceinline__ float4 merge_warps(const Sums<DH, HEADS>& s, int h, int d, float& m, float& l) {
  float f[PA_WARPS];
  m = -INFINITY;
#pragma unroll
  for (int w = 0; w < PA_WARPS; ++w) m = fmaxf(m, s.m[w][h]);
  const float u = m == -INFINITY ? 0.f : m;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  l = 0.f;
#pragma unroll
  for (int w = 0; w < PA_WARPS; ++w) {
    f[w] = exp2f(s.m[w][h] - u);
    l += s.l[w][h] * f[w];
    const float4 x = *reinterpret_cast<const float4*>(&s.o[w][h][d]);
    o = make_float4(o.x + x.x * f[w], o.y + x.y * f[w], o.z + x.z * f[w], o.w + x.w * f[w]);
  }
  return o;
}
// What a sum of weights is divided by, as a factor.  (A row without keys: zeros; its lse is the logarithm of nothing.)
__device__ __forceinline__ float one_over(float l) { return l > 0.f || l != l ? 1.f / l : 0.f; }
template <typename T>
__device__ __forceinline__ void store_out(const PagedParams& p, size_t row, int d, int dh, float x) {
  if constexpr (sizeof(T) == 2) reinterpret_cast<bf16*>(p.out)[row * dh + d] = __float2bfloat16_rn(x);
  else reinterpret_cast<float*>(p.out)[row * dh + d] = x;
}
template <typename T>
__device__ __forceinline__ void store_out(const PagedParams& p, size_t row, int d, int dh, float4 x) {
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(p.out) + row * dh + d) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
  else
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(p.out) + row * dh + d) = x;
}
__device__ __forceinline__ void store_lse(const PagedParams& p, size_t row, float m, float l) {
  if (p.lse) p.lse[row] = (m + log2f(l)) * kLn2;
}

// A piece of a unit: the items from item0 up to item1, of which a warp takes every stride-th, for these of the query heads.
struct Piece {
  Span sp;
  int b, kvh, head0, heads, item0, item1, stride;
  PageRef ahead;                  // of this lane's item among the warp's first 32
};
__device__ __forceinline__ int warp_item(const Piece& c, int i) { return c.item0 + (int)(threadIdx.x >> 5) + i * c.stride; }
// The pages that a warp goes through, looked up 32 at a time.
struct Walk {
  int i = 0, mine, pages_l = -1, at_l = -1;
  __device__ __forceinline__ explicit Walk(const Piece& c) : mine(max(0, (c.item1 - warp_item(c, 0) + c.stride - 1) / c.stride)) {}
  // the next one that there is something to read of, or {-1, -1}
  __device__ __forceinline__ PageRef next(const PagedParams& p, const Piece& c) {
    const int lane = threadIdx.x & 31;
    PageRef r{-1, -1};
    while (i < mine) {
      if (i % 32 == 0) {
        const PageRef l = i == 0 ? c.ahead : page_ref(p, c.sp.first, c.b, c.kvh, warp_item(c, i + lane));
        pages_l = l.page;
        at_l = i + lane < mine && (unsigned)l.page < (unsigned)((c.sp.hi + CERB_PAGE - 1) / CERB_PAGE) ? l.at : -1;
      }
      r.page = __shfl_sync(0xffffffffu, pages_l, i % 32);
      r.at = __shfl_sync(0xffffffffu, at_l, i % 32);
      ++i;
      if (r.at >= 0) break;
    }
    return r;
  }
};

__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}


// bf16.  Both products have the keys (of K q: 16 keys; of V p: Dh) on the MMA's 16 rows and the heads, NT groups of eight, on its columns: S^T = K q^T,
// out^T = V^T P^T.  The order of the k positions of a product is free as long as both operands have the same, so a lane's 16
// bytes of a key row (8 consecutive elements) are what it needs of two MMAs, and what it loads of the values, 8 elements of each of four keys, is
// interleaved into fragments by byte permutes.  S^T's sums become P^T's fragments by 8 x 8 transpositions of 16-bit elements.
// P enters the second product as two bf16 terms, itself rounded and what that leaves, as in tree attention: a weight is off by at most 2^-16 of itself, and the sum l is that of the unrounded
// ones; scores, maxima, sums and outputs are fp32.  (With one term a weight is off by up to 2^-8.  The second costs, us with one / two: 64 sequences of up to 8192 tokens 193.8 / 194.1, one of 1000
// 5.6 / 5.7, 128 of 2000 with heads of 64 55.4 / 56.4, 16 of 4096 with 16 heads to a unit 26.9 / 27.4, 16 of 32768 with 16 / 64 heads on one KV head 54.7 / 56.1
// and 154.5 / 161.6, 24 selections of 128 pages 65.6 / 65.9 with the selection.  The figures below that compare forms were taken with one.)
// A warp takes KP pages at a time, 8 KB of keys and values, and has the next AHEAD times as many on their way.
template <int DH, int NT, int AHEAD>
__device__ __forceinline__ void attend_bf16(const PagedParams& p, const Piece& c, Sums<DH, 8 * NT>& sums) {
  constexpr int KC = DH / 32, VH = DH / 64, KP = 128 / DH;               // chunks of a key row, halves of a value row, pages at a time
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const bf16* kp = reinterpret_cast<const bf16*>(p.k_pool) + (size_t)c.kvh * CERB_PAGE * DH + g * DH + t * 8;
  const bf16* vp = reinterpret_cast<const bf16*>(p.v_pool) + (size_t)c.kvh * CERB_PAGE * DH + 2 * t * DH + g * 8;
  const size_t page_elems = (size_t)p.Hk * CERB_PAGE * DH;
  Walk walk(c);
  uint4 kk[AHEAD][KP][2][KC], vv[AHEAD][KP][4][VH];
  auto load_k = [&](uint4 (&k)[KP][2][KC], const PageRef (&r)[KP]) {
#pragma unroll
    for (int a = 0; a < KP; ++a)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int j = 0; j < KC; ++j) k[a][e][j] = KP == 1 || r[a].at >= 0 ? ld16(kp + r[a].at * page_elems + e * 8 * DH + 32 * j) : make_uint4(0, 0, 0, 0);
  };
  auto load_v = [&](uint4 (&v)[KP][4][VH], const PageRef (&r)[KP]) {
#pragma unroll
    for (int a = 0; a < KP; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < VH; ++j)
          v[a][e][j] = KP == 1 || r[a].at >= 0 ? ld16(vp + r[a].at * page_elems + ((e & 1) + 8 * (e >> 1)) * DH + 64 * j) : make_uint4(0, 0, 0, 0);
  };
  PageRef ahead[AHEAD][KP];
#pragma unroll
  for (int x = 0; x < AHEAD; ++x) {
#pragma unroll
    for (int a = 0; a < KP; ++a) ahead[x][a] = walk.next(p, c);
    if (ahead[x][0].at >= 0) { load_k(kk[x], ahead[x]); load_v(vv[x], ahead[x]); }
  }
  uint4 q[NT][KC];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < KC; ++j)
      q[n][j] = 8 * n + g < c.heads
                    ? *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(p.q) + (size_t)c.b * p.q_row + (size_t)(c.head0 + 8 * n + g) * p.q_head + 32 * j + 8 * t)
                    : make_uint4(0, 0, 0, 0);
  float o[NT][4 * VH][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n][0] = m[n][1] = -INFINITY;
    l[n][0] = l[n][1] = 0.f;
#pragma unroll
    for (int d = 0; d < 4 * VH; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n][d][e] = 0.f;
  }
  while (ahead[0][0].at >= 0) {
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) {
      PageRef (&now)[KP] = ahead[x];
      uint4 (&k)[KP][2][KC] = kk[x];
      uint4 (&v)[KP][4][VH] = vv[x];
      if (now[0].at < 0) break;                                            // (and none behind it)
      PageRef then[KP];
#pragma unroll
      for (int a = 0; a < KP; ++a) then[a] = walk.next(p, c);
      float s[KP][NT][4];
#pragma unroll
      for (int a = 0; a < KP; ++a)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          // (two accumulators: the tensor cores cut a sum off at every step)
          float a0[4] = {0.f, 0.f, 0.f, 0.f}, a1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < KC; ++j) {
            mma_16816(a0, k[a][0][j].x, k[a][1][j].x, k[a][0][j].y, k[a][1][j].y, q[n][j].x, q[n][j].y);
            mma_16816(a1, k[a][0][j].z, k[a][1][j].z, k[a][0][j].w, k[a][1][j].w, q[n][j].z, q[n][j].w);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) s[a][n][e] = (a0[e] + a1[e]) * p.scale_log2;
        }
      if (then[0].at >= 0) load_k(k, then);
#pragma unroll
      for (int a = 0; a < KP; ++a) {
        const int row0 = now[a].at >= 0 ? now[a].page * CERB_PAGE : c.sp.hi;
        if (row0 < c.sp.lo || row0 + CERB_PAGE > c.sp.hi) {
          // the ends: whatever lies outside counts nothing, and is nothing (it may be infinite)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = row0 + g + 8 * (e >> 1);
              if (r < c.sp.lo || r >= c.sp.hi) s[a][n][e] = -INFINITY;
            }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = row0 + 2 * t + (e & 1) + 8 * (e >> 1);
            if (r < c.sp.lo || r >= c.sp.hi)
#pragma unroll
              for (int j = 0; j < VH; ++j) v[a][e][j] = make_uint4(0, 0, 0, 0);
          }
        }
      }
      uint32_t pb[KP][NT][2], pl[KP][NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float mx[2] = {fmaxf(s[0][n][0], s[0][n][2]), fmaxf(s[0][n][1], s[0][n][3])};
#pragma unroll
        for (int a = 1; a < KP; ++a)
#pragma unroll
          for (int e = 0; e < 2; ++e) mx[e] = fmaxf(mx[e], fmaxf(s[a][n][e], s[a][n][e + 2]));
#pragma unroll
        for (int w = 4; w < 32; w <<= 1)
#pragma unroll
          for (int e = 0; e < 2; ++e) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], w));
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          mx[e] = fmaxf(mx[e], m[n][e]);
          const float u = mx[e] == -INFINITY ? 0.f : mx[e];
          f[e] = exp2f(m[n][e] - u);
          m[n][e] = mx[e];
          l[n][e] *= f[e];
#pragma unroll
          for (int a = 0; a < KP; ++a) {
            s[a][n][e] = exp2f(s[a][n][e] - u);
            s[a][n][e + 2] = exp2f(s[a][n][e + 2] - u);
            l[n][e] += s[a][n][e] + s[a][n][e + 2];
          }
        }
        if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
          for (int d = 0; d < 4 * VH; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][d][e] *= f[e & 1];
        }
#pragma unroll
        for (int a = 0; a < KP; ++a) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t hi = pack_bf16(s[a][n][2 * e], s[a][n][2 * e + 1]);
            pb[a][n][e] = transpose8x8(hi);
            pl[a][n][e] = transpose8x8(pack_bf16(s[a][n][2 * e] - __uint_as_float(hi << 16), s[a][n][2 * e + 1] - __uint_as_float(hi & 0xffff0000u)));
          }
        }
      }
#pragma unroll
      for (int a = 0; a < KP; ++a)
#pragma unroll
        for (int j = 0; j < VH; ++j) {
          const uint32_t x[4][4] = {{v[a][0][j].x, v[a][0][j].y, v[a][0][j].z, v[a][0][j].w}, {v[a][1][j].x, v[a][1][j].y, v[a][1][j].z, v[a][1][j].w},
                                    {v[a][2][j].x, v[a][2][j].y, v[a][2][j].z, v[a][2][j].w}, {v[a][3][j].x, v[a][3][j].y, v[a][3][j].z, v[a][3][j].w}};
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t a0 = __byte_perm(x[0][d], x[1][d], 0x5410), a1 = __byte_perm(x[0][d], x[1][d], 0x7632);
            const uint32_t a2 = __byte_perm(x[2][d], x[3][d], 0x5410), a3 = __byte_perm(x[2][d], x[3][d], 0x7632);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma_16816(o[n][4 * j + d], a0, a1, a2, a3, pb[a][n][0], pb[a][n][1]);
              mma_16816(o[n][4 * j + d], a0, a1, a2, a3, pl[a][n][0], pl[a][n][1]);
            }
          }
        }
      if (then[0].at >= 0) load_v(v, then);
#pragma unroll
      for (int a = 0; a < KP; ++a) now[a] = then[a];
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], w);
      const int h = 8 * n + 2 * t + e;
      if (g == 0) { sums.m[warp][h] = m[n][e]; sums.l[warp][h] = l[n][e]; }
      // accumulator d of half j: rows g and g + 8 of the MMA are the elements 2d and 2d + 1 of the lane's eight
#pragma unroll
      for (int d = 0; d < 4 * VH; ++d)
        *reinterpret_cast<float2*>(&sums.o[warp][h][(d >> 2) * 64 + 8 * g + 2 * (d & 3)]) = make_float2(o[n][d][e], o[n][d][e + 2]);
    }
}

// fp32, one or two heads to a unit, or four of 128: plain FMA.  (One head to a KV head: 117 MB in 21 us, 5.6 TB/s; 16 sequences of 8192 tokens, 4 heads on each of 8, 1074 MB: 164 us, 6.5 TB/s.)
// A lane owns DH / 32 elements of every key and value, a warp takes KEYS keys at a time for up to GH heads and has the next ones on their way.
// The lanes' KEYS x GH partial sums meet by halving, after which each lane has the scores of few keys to take the exponential of; the weights come back by
// shuffles.
template <int DH, int GH>
__device__ __forceinline__ void attend_f32(const PagedParams& p, const Piece& c, Sums<DH, GH>& sums) {
  constexpr int E = DH / 32, KEYS = DH == 64 && GH <= 2 ? 16 : 8, STEPS = CERB_PAGE / KEYS;
  constexpr int NV = KEYS * GH, R = NV >= 32 ? NV / 32 : 1, REP = NV >= 32 ? 1 : 32 / NV, LPH = 32 / GH;   // sums of a lane at the end, lanes with the same one; lanes of a head
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const size_t page_elems = (size_t)p.Hk * CERB_PAGE * DH;
  const float* kp = reinterpret_cast<const float*>(p.k_pool) + (size_t)c.kvh * CERB_PAGE * DH + lane * E;
  const float* vp = reinterpret_cast<const float*>(p.v_pool) + (size_t)c.kvh * CERB_PAGE * DH + lane * E;
  struct Row {
    float x[E];
  };
  auto load_rows = [&](Row (&r)[KEYS], const float* src) {
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
      if constexpr (E == 4)
        asm volatile("ld.global.L1::no_allocate.L2::256B.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(r[j].x[0]), "=f"(r[j].x[1]), "=f"(r[j].x[2]), "=f"(r[j].x[3]) : "l"(src + j * DH) : "memory");
      else
        asm volatile("ld.global.L1::no_allocate.L2::256B.v2.f32 {%0, %1}, [%2];" : "=f"(r[j].x[0]), "=f"(r[j].x[1]) : "l"(src + j * DH) : "memory");
    }
  };
  // this warp's steps: the parts of its pages that have a live row
  Walk walk(c);
  int step = STEPS;
  PageRef page{-1, -1};
  struct Step {
    int row0;
    long long at;                                                        // element of the pools, -1: none
  };
  auto next = [&]() {
    for (;;) {
      if (step == STEPS) {
        page = walk.next(p, c);
        if (page.at < 0) return Step{0, -1};
        step = 0;
      }
      const int row0 = page.page * CERB_PAGE + step * KEYS;
      const long long at = (long long)(page.at * page_elems) + step * KEYS * DH;
      ++step;
      if (row0 < c.sp.hi && row0 + KEYS > c.sp.lo) return Step{row0, at};
    }
  };
  Row k[KEYS], v[KEYS];
  Step now = next();
  if (now.at >= 0) { load_rows(k, kp + now.at); load_rows(v, vp + now.at); }
  float q[GH][E], o[GH][E];
#pragma unroll
  for (int h = 0; h < GH; ++h)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[h][e] = h < c.heads ? reinterpret_cast<const float*>(p.q)[(size_t)c.b * p.q_row + (size_t)(c.head0 + h) * p.q_head + lane * E + e] : 0.f;
      o[h][e] = 0.f;
    }
  float m = -INFINITY, l = 0.f;                                          // of head lane / LPH
  while (now.at >= 0) {
    const Step then = next();
    float s[NV];                                                         // [head][key]
#pragma unroll
    for (int h = 0; h < GH; ++h)
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) x = fmaf(q[h][e], k[j].x[e], x);
        s[h * KEYS + j] = x;
      }
    if (then.at >= 0) load_rows(k, kp + then.at);
    halve_sums(s, lane);
    const bool ends = now.row0 < c.sp.lo || now.row0 + KEYS > c.sp.hi;
    float mx = m;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] *= p.scale_log2;
      const int row = now.row0 + (lane / REP * R + r) % KEYS;
      if (ends && (row < c.sp.lo || row >= c.sp.hi)) s[r] = -INFINITY;
      mx = fmaxf(mx, s[r]);
    }
    if (ends) {
#pragma unroll
      for (int j = 0; j < KEYS; ++j)
        if (now.row0 + j < c.sp.lo || now.row0 + j >= c.sp.hi)
#pragma unroll
          for (int e = 0; e < E; ++e) v[j].x[e] = 0.f;
    }
#pragma unroll
    for (int w = 1; w < LPH; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
    const float u = mx == -INFINITY ? 0.f : mx, a = exp2f(m - u);
    m = mx;
    l *= a;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = exp2f(s[r] - u);
      if (lane % REP == 0) l += s[r];
    }
#pragma unroll
    for (int h = 0; h < GH; ++h) {
      const float ah = __shfl_sync(0xffffffffu, a, h * LPH);
#pragma unroll
      for (int e = 0; e < E; ++e) o[h][e] *= ah;
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        const int idx = h * KEYS + j;
        const float w = __shfl_sync(0xffffffffu, s[idx % R], idx / R * REP);
#pragma unroll
        for (int e = 0; e < E; ++e) o[h][e] = fmaf(w, v[j].x[e], o[h][e]);
      }
    }
    if (then.at >= 0) load_rows(v, vp + then.at);
    now = then;
  }
#pragma unroll
  for (int w = 1; w < LPH; w <<= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
  if (lane % LPH == 0) { sums.m[warp][lane / LPH] = m; sums.l[warp][lane / LPH] = l; }
#pragma unroll
  for (int h = 0; h < GH; ++h)
#pragma unroll
    for (int e = 0; e < E; ++e) sums.o[warp][h][lane * E + e] = o[h][e];
}

// fp32, many heads to a unit: FMA on pairs.  A warp takes a page at a time and has the next one on its way.  What a lane reads of shared memory costs the SM 32 lanes' bytes
// at 128 a cycle, the same address or not; so few bytes a lane decide the split.  Scores: lanes 8g .. 8g + 7 have keys g, g + 4, g + 8, g + 12, an eighth of the elements each (16 bytes of
// every 128), the queries come out of shared memory, four chains of sums to a key and head keep the roundings in a row at Dh / 32 + 5.  Their GH x 4 sums meet by
// halving, so that a lane has GH / 2 scores of one head.  Weights go through shared memory, two heads a pair; outputs: four columns to a lane
// (heads of 64: every other key to each half of the warp).
// 16 sequences of 8192 tokens, 8 heads of 128 on each of 8, 1074 MB: 170 us, 6.3 TB/s; 100 of 1600, 8 heads of 64, 655 MB: 120, 5.5 TB/s; 16 heads, two units, each of which reads
// the keys and values: 100 of 1600 220, 100 of 1280 185.
// (With the lanes' way of the other fp32 form, 62 shuffles and 64 broadcasts for 8 keys of 8 heads: 216, 210, 326.  With a quarter of a key to a lane and weights twice in shared memory, the data
// pipe of shared memory and L1 71 % busy: 191, 130, 201.  Four heads of 64 on each of 8, 16 x 9600 tokens: 127 -> 101 us, at the copy rate; four heads of 128: at the copy rate either way.)
template <int DH, int GH>
__device__ __forceinline__ void attend_f32_many(const PagedParams& p, const Piece& c, Sums<DH, GH>& sums) {
  constexpr int CH = DH / 32, R = GH / 2, SIDES = 128 / DH, VK = CERB_PAGE / SIDES;
  __shared__ alignas(16) float s_p[PA_WARPS][CERB_PAGE][GH], s_a[PA_WARPS][GH];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 3, t = lane & 7, side = lane / (DH / 4), col = lane % (DH / 4) * 4;
  const int head = t * GH / 8, key0 = g + 4 * R * (t % (8 / GH));         // of the lane's scores
  const size_t page_elems = (size_t)p.Hk * CERB_PAGE * DH;
  const float* kp = reinterpret_cast<const float*>(p.k_pool) + (size_t)c.kvh * CERB_PAGE * DH + g * DH + 4 * t;
  const float* vp = reinterpret_cast<const float*>(p.v_pool) + (size_t)c.kvh * CERB_PAGE * DH + side * DH + col;
  f32x2 k[4][CH][2];
  float4 v[VK];
  auto load_k = [&](const PageRef& r) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < CH; ++i)
        asm volatile("ld.global.L1::no_allocate.L2::256B.v2.b64 {%0, %1}, [%2];"
                     : "=l"(k[e][i][0]), "=l"(k[e][i][1]) : "l"(kp + r.at * page_elems + e * 4 * DH + 32 * i) : "memory");
  };
  auto load_v = [&](const PageRef& r) {
#pragma unroll
    for (int j = 0; j < VK; ++j)
      asm volatile("ld.global.L1::no_allocate.L2::256B.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(v[j].x), "=f"(v[j].y), "=f"(v[j].z), "=f"(v[j].w) : "l"(vp + r.at * page_elems + j * SIDES * DH) : "memory");
  };
  Walk walk(c);
  auto next = [&]() {
    for (;;) {
      const PageRef r = walk.next(p, c);
      if (r.at < 0 || (r.page * CERB_PAGE < c.sp.hi && (r.page + 1) * CERB_PAGE > c.sp.lo)) return r;
    }
  };
  PageRef now = next();
  if (now.at >= 0) { load_k(now); load_v(now); }
  // the queries, where the outputs go at the end
  float* s_q = &sums.o[warp][0][0];
  for (int i = 4 * lane; i < GH * DH; i += 4 * 32) {
    const int h = i / DH;
    *reinterpret_cast<float4*>(s_q + i) =
        h < c.heads ? *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.q) + (size_t)c.b * p.q_row + (size_t)(c.head0 + h) * p.q_head + i % DH)
                    : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __syncwarp();
  f32x2 o[GH / 2][4];                                                    // [pair of heads][column]
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int h = 0; h < GH / 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[h][e] = 0;
  while (now.at >= 0) {
    const PageRef then = next();
    float s[4 * GH];                                                     // [head][key]
#pragma unroll
    for (int h = 0; h < GH; ++h) {
      f32x2 x[4][2];
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(s_q + h * DH + 32 * i + 4 * t);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e][0] = i == 0 ? mul2(q.x, k[e][i][0]) : fma2(q.x, k[e][i][0], x[e][0]);
          x[e][1] = i == 0 ? mul2(q.y, k[e][i][1]) : fma2(q.y, k[e][i][1], x[e][1]);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 y = parts_of(add2(x[e][0], x[e][1]));
        s[4 * h + e] = y.x + y.y;
      }
    }
    if (then.at >= 0) load_k(then);
#pragma unroll
    for (int w = 4, n = 2 * GH; w > 0; w >>= 1, n >>= 1)
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const bool up = lane & w;
        const float send = up ? s[i] : s[i + n], keep = up ? s[i + n] : s[i];
        s[i] = keep + __shfl_xor_sync(0xffffffffu, send, w);
      }
    // s[i]: key key0 + 4 i
    const int row0 = now.page * CERB_PAGE;
    const bool ends = row0 < c.sp.lo || row0 + CERB_PAGE > c.sp.hi;
    float mx = m;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      s[i] *= p.scale_log2;
      const int row = row0 + key0 + 4 * i;
      if (ends && (row < c.sp.lo || row >= c.sp.hi)) s[i] = -INFINITY;
      mx = fmaxf(mx, s[i]);
    }
#pragma unroll
    for (int w = 8; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
    if constexpr (GH == 4) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    const float u = mx == -INFINITY ? 0.f : mx, a = exp2f(m - u);
    const bool moved = __any_sync(0xffffffffu, a != 1.f);
    m = mx;
    l *= a;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float x = exp2f(s[i] - u);
      l += x;
      s_p[warp][key0 + 4 * i][head] = x;
    }
    if (moved && key0 == 0) s_a[warp][head] = a;
    if (ends) {
#pragma unroll
      for (int j = 0; j < VK; ++j) {
        const int row = row0 + j * SIDES + side;
        if (row < c.sp.lo || row >= c.sp.hi) v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
    __syncwarp();
    if (moved) {
#pragma unroll
      for (int h = 0; h < GH / 2; ++h) {
        const f32x2 x = *reinterpret_cast<const f32x2*>(&s_a[warp][2 * h]);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[h][e] = mul2(o[h][e], x);
      }
    }
#pragma unroll
    for (int j = 0; j < VK; ++j) {
      const f32x2 x[4] = {twice(v[j].x), twice(v[j].y), twice(v[j].z), twice(v[j].w)};
#pragma unroll
      for (int h = 0; h < GH / 2; h += 2) {
        const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(&s_p[warp][j * SIDES + side][2 * h]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[h][e] = fma2(w.x, x[e], o[h][e]);
          o[h + 1][e] = fma2(w.y, x[e], o[h + 1][e]);
        }
      }
    }
    if (then.at >= 0) load_v(then);
    __syncwarp();
    now = then;
  }
#pragma unroll
  for (int w = 8; w < 32; w <<= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
  if constexpr (GH == 4) l += __shfl_xor_sync(0xffffffffu, l, 1);
  if (key0 == 0) { sums.m[warp][head] = m; sums.l[warp][head] = l; }
#pragma unroll
  for (int h = 0; h < GH / 2; ++h) {
    float2 x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (SIDES == 2) o[h][e] = add2(o[h][e], __shfl_xor_sync(0xffffffffu, o[h][e], 16));
      x[e] = parts_of(o[h][e]);
    }
    if (side) continue;
    *reinterpret_cast<float4*>(&sums.o[warp][2 * h][col]) = make_float4(x[0].x, x[1].x, x[2].x, x[3].x);
    *reinterpret_cast<float4*>(&sums.o[warp][2 * h + 1][col]) = make_float4(x[0].y, x[1].y, x[2].y, x[3].y);
  }
}

template <typename T, int DH, int HEADS, int AHEAD = 1>
__device__ __forceinline__ void attend(const PagedParams& p, const Piece& c, Sums<DH, HEADS>& sums) {
  if constexpr (sizeof(T) == 2) attend_bf16<DH, HEADS / 8, AHEAD>(p, c, sums);
  else if constexpr (HEADS == 8 || (HEADS == 4 && DH == 64)) attend_f32_many<DH, HEADS>(p, c, sums);
  else attend_f32<DH, HEADS>(p, c, sums);
}

// None of the three forms lets the next kernel be scheduled before it ends: waiting CTAs take the places of those that end first, and then run on crowded SMs while others idle.
// (us a pass that follows another, with an early release / without: 64 sequences of up to 8192 tokens 192 / 189.7, a window of 16001 40.4 / 38.8, 123 MB of fp32 in clusters 23.2 / 21.7, 32 units
// of 60 pages 7.3 / 6.5, 1024 of 16 27.8 / 24.6; one sequence of 1000 tokens 5.4 / 5.5.)
// CTAs that fit an SM, as the kernels' registers allow.
// (fp32, 8 heads of 64, 2 / 3 / 4: 100 sequences of 100 pages 126 / 120 / 154 us.)
template <typename T, int DH, int HEADS>
constexpr int ctas_per_sm() { return sizeof(T) == 2 ? (HEADS == 8 ? 3 : 2) : HEADS <= 2 ? 4 : HEADS == 4 || DH == 64 ? 3 : 2; }

// Every CTA a share.
template <typename T, int DH, int HEADS>
__global__ void __launch_bounds__(PA_WARPS * 32, ctas_per_sm<T, DH, HEADS>()) paged_attn_kernel(const PagedParams p) {
  __shared__ Sums<DH, HEADS> sums;
  griddep_wait();
  const long long uh = (long long)p.Hk * p.units_h;
  const Share sh = share_of(p.B, [&](int b) { return span_of(p, b).items * uh; }, blockIdx.x, gridDim.x, p.min_share, p.B * uh);
  // sequences without anything to look at
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    if (span_of(p, b).items) continue;
    for (size_t i = threadIdx.x; i < (size_t)p.H * DH; i += PA_WARPS * 32) store_out<T>(p, (size_t)b * p.H + i / DH, (int)(i % DH), DH, 0.f);
    for (int i = threadIdx.x; i < p.H; i += PA_WARPS * 32) store_lse(p, (size_t)b * p.H + i, -INFINITY, 0.f);
    if (p.by_unit)
      for (int i = threadIdx.x; i < uh; i += PA_WARPS * 32) p.meta[b * uh + i] = make_int4(0, 0, 0, 0);
  }
  bool left = !p.by_unit;                                                // this CTA's join is still to be said
  Piece c;
  c.b = sh.b;
  c.stride = PA_WARPS;
  long long off = sh.off;
  for (long long at = sh.begin; at < sh.end;) {
    c.sp = span_of(p, c.b);
    if (off >= c.sp.items * uh) {                                        // (the next one that has items)
      ++c.b;
      off = 0;
      continue;
    }
    const int items = c.sp.items;
    const int u = off >> 32 ? (int)(off / items) : (int)((unsigned)off / (unsigned)items);
    c.item0 = (int)(off - (long long)u * items);
    const int n = (int)min((long long)(items - c.item0), sh.end - at);
    c.item1 = c.item0 + n;
    c.kvh = u / p.units_h;
    c.ahead = page_ref(p, c.sp.first, c.b, c.kvh, warp_item(c, threadIdx.x & 31));
    const int part = u - c.kvh * p.units_h, unit = (int)(c.b * uh) + u;
    c.head0 = c.kvh * p.G + part * HEADS;
    c.heads = min(HEADS, p.G - part * HEADS);
    const int slot = 2 * (int)blockIdx.x + (at != sh.begin);             // where a part goes: a CTA has two at most, its first piece and its last
    // (a unit whose first part is this one: of those a CTA has one at most, the last of its pieces)
    if (c.item0 == 0 && (p.by_unit || n < items)) {
      if (threadIdx.x == 0)
        p.meta[p.by_unit ? unit : blockIdx.x] = make_int4(unit, slot, n == items ? 1 : (int)((at + items - 1) / sh.size - blockIdx.x) + 1, 0);
      left = false;
    }
    attend<T, DH, HEADS>(p, c, sums);
    __syncthreads();
    for (int i = 4 * threadIdx.x; i < c.heads * DH; i += 4 * PA_WARPS * 32) {
      const int h = i / DH, d = i % DH;
      float m, l;
      const float4 o = merge_warps(sums, h, d, m, l);
      if (n < items) {
        const size_t to = (size_t)slot * HEADS + h;
        *reinterpret_cast<float4*>(p.part_o + to * DH + d) = o;
        if (d == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * to) = make_float2(m, l);
      } else {
        const float r = one_over(l);
        const size_t row = (size_t)c.b * p.H + c.head0 + h;
        store_out<T>(p, row, d, DH, make_float4(o.x * r, o.y * r, o.z * r, o.w * r));
        if (d == 0) store_lse(p, row, m, l);
      }
    }
    __syncthreads();
    at += n;
    off += n;
  }
  if (left && threadIdx.x == 0) p.meta[blockIdx.x] = make_int4(0, 0, 0, 0);
}

// Every unit a cluster, which meets in its CTAs' shared memory: each CTA joins a part of the outputs, sent to it by all.
template <typename T, int DH, int HEADS, int AHEAD>
__global__ void __launch_bounds__(PA_WARPS * 32, AHEAD == 1 ? ctas_per_sm<T, DH, HEADS>() : 2) paged_attn_cluster_kernel(const PagedParams p) {
  __shared__ Sums<DH, HEADS> sums;
  __shared__ alignas(16) float s_o[HEADS * DH];                          // [CTA][its part of the outputs]
  __shared__ alignas(16) float2 s_ml[HEADS][PA_CLUSTER];
  __shared__ float s_f[PA_CLUSTER][HEADS];                               // weight of a CTA's sums in a head's result
  const int n = p.together, rank = blockIdx.x % n, unit = blockIdx.x / n;
  cluster_start_arrive();
  const int part = unit % p.units_h;
  Piece c;
  c.kvh = unit / p.units_h % p.Hk;
  c.b = unit / p.units_h / p.Hk;
  c.head0 = c.kvh * p.G + part * HEADS;
  c.heads = min(HEADS, p.G - part * HEADS);
  griddep_wait();
  // (the items are dealt out one by one, so that the first ones can be looked up before the length is known)
  c.item0 = rank * PA_WARPS;
  c.stride = n * PA_WARPS;
  if (p.window == 0 || p.sel) c.ahead = page_ref(p, 0, c.b, c.kvh, warp_item(c, threadIdx.x & 31));
  c.sp = span_of(p, c.b);
  if (p.window > 0 && !p.sel) c.ahead = page_ref(p, c.sp.first, c.b, c.kvh, warp_item(c, threadIdx.x & 31));
  c.item1 = c.sp.items;
  const int own = HEADS * DH / n;
  attend<T, DH, HEADS, AHEAD>(p, c, sums);
  __syncthreads();
  cluster_start_wait();                                                  // every CTA of the cluster runs
  for (int i = 4 * threadIdx.x; i < c.heads * DH; i += 4 * PA_WARPS * 32) {
    float m, l;
    const int h = i / DH, d = i % DH, to = i / own;                      // (a CTA's part of the outputs is a multiple of four columns)
    const float4 o = merge_warps(sums, h, d, m, l);
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(mapa_u32(smem_u32(&s_o[rank * own + i - to * own]), to)), "f"(o.x), "f"(o.y), "f"(o.z),
                 "f"(o.w) : "memory");
    // (the maximum and the sum of a head: to all, one each from the threads of its first columns)
    if (d / 4 < n)
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(mapa_u32(smem_u32(&s_ml[h][rank]), d / 4)), "f"(m), "f"(l) : "memory");
  }
  cluster_start_arrive();
  cluster_start_wait();                                                  // ... and has sent its sums
  // the heads of this CTA's part, a CTA of the cluster to a lane
  const int h0 = rank * own / DH, h1 = min(c.heads, (rank * own + own - 1) / DH + 1);
  for (int h = h0 + (threadIdx.x >> 5); h < h1; h += PA_WARPS) {
    const int lane = threadIdx.x & 31;
    const float2 x = lane < n ? s_ml[h][lane] : make_float2(-INFINITY, 0.f);
    float m = x.x;
#pragma unroll
    for (int w = PA_CLUSTER / 2; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
    const float f = exp2f(x.x - (m == -INFINITY ? 0.f : m));
    float l = x.y * f;
#pragma unroll
    for (int w = PA_CLUSTER / 2; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
    if (lane < n) s_f[lane][h] = f * one_over(l);
    if (lane == 0 && rank * own <= h * DH) store_lse(p, (size_t)c.b * p.H + c.head0 + h, m, l);
  }
  __syncthreads();
  for (int j = threadIdx.x; j < own; j += PA_WARPS * 32) {
    const int i = rank * own + j, h = i / DH;
    if (h >= c.heads) break;
    float o = 0.f;
#pragma unroll 4
    for (int r = 0; r < n; ++r) o = fmaf(s_f[r][h], s_o[r * own + j], o);
    store_out<T>(p, (size_t)c.b * p.H + c.head0 + h, i % DH, DH, o);
  }
}

// Every unit a warp, for many short sequences: nothing to meet, no barrier.
template <typename T, int DH, int HEADS>
__global__ void __launch_bounds__(PA_WARPS * 32, ctas_per_sm<T, DH, HEADS>()) paged_attn_warp_kernel(const PagedParams p) {
  __shared__ Sums<DH, HEADS> sums;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * PA_WARPS + warp;
  griddep_wait();
  const int part = (int)(unit % p.units_h);
  Piece c;
  c.kvh = (int)(unit / p.units_h % p.Hk);
  const long long b = unit / p.units_h / p.Hk;
  if (b >= p.B) return;
  c.b = (int)b;
  c.head0 = c.kvh * p.G + part * HEADS;
  c.heads = min(HEADS, p.G - part * HEADS);
  c.item0 = -warp;                                                       // (all of the items are this warp's)
  c.stride = 1;
  if (p.window == 0 || p.sel) c.ahead = page_ref(p, 0, c.b, c.kvh, lane);
  c.sp = span_of(p, c.b);
  if (p.window > 0 && !p.sel) c.ahead = page_ref(p, c.sp.first, c.b, c.kvh, lane);
  c.item1 = c.sp.items;
  attend<T, DH, HEADS>(p, c, sums);
  __syncwarp();
  for (int i = 4 * lane; i < c.heads * DH; i += 4 * 32) {
    const int h = i / DH, d = i % DH;
    const size_t row = (size_t)c.b * p.H + c.head0 + h;
    const float4 o = *reinterpret_cast<const float4*>(&sums.o[warp][h][d]);
    const float r = one_over(sums.l[warp][h]);
    store_out<T>(p, row, d, DH, make_float4(o.x * r, o.y * r, o.z * r, o.w * r));
    if (d == 0) store_lse(p, row, sums.m[warp][h], sums.l[warp][h]);
  }
}

// The parts of a unit as one.  A warp takes a head (heads_y of them per CTA) and every groups-th part.
template <typename T, int DH>
__global__ void __launch_bounds__(1024) paged_join_kernel(const PagedParams p, int heads_unit, int heads_y) {
  constexpr int E = DH / 32;
  struct alignas(4 * E) Cols {
    float x[E];
  };
  __shared__ Cols s_o[32][32];
  __shared__ float s_m[32], s_l[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, groups = blockDim.x / 32 / heads_y, grp = warp / heads_y;
  const int h = blockIdx.y * heads_y + warp % heads_y;
  griddep_wait();
  griddep_launch();
  const int4 j = p.meta[blockIdx.x];
  if (j.z <= 1) return;
  const int unit = j.x, part = unit % p.units_h, kvh = unit / p.units_h % p.Hk, b = unit / p.units_h / p.Hk;
  const bool live = part * heads_unit + h < p.G;
  float m = -INFINITY, l = 0.f;
  Cols o;
#pragma unroll
  for (int e = 0; e < E; ++e) o.x[e] = 0.f;
  // (the first may be the second part of its CTA, the others are the first ones of the CTAs that follow)
#pragma unroll 8
  for (int i = live ? grp : j.z; i < j.z; i += groups) {
    const size_t at = (size_t)(i ? (j.y & ~1) + 2 * i : j.y) * heads_unit + h;
    const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * at);
    const Cols x = *reinterpret_cast<const Cols*>(p.part_o + at * DH + lane * E);
    const float mx = fmaxf(m, ml.x), u = mx == -INFINITY ? 0.f : mx;
    const float f = exp2f(m - u), g = exp2f(ml.x - u);
    l = l * f + ml.y * g;
#pragma unroll
    for (int e = 0; e < E; ++e) o.x[e] = o.x[e] * f + x.x[e] * g;
    m = mx;
  }
  if (groups > 1) {
    s_o[warp][lane] = o;
    if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
    __syncthreads();
    if (grp) return;
    for (int i = 1; i < groups; ++i) m = fmaxf(m, s_m[warp + i * heads_y]);
    const float u = m == -INFINITY ? 0.f : m;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) o.x[e] = 0.f;
    for (int i = 0; i < groups; ++i) {
      const int w = warp + i * heads_y;
      const float f = exp2f(s_m[w] - u);
      l += s_l[w] * f;
      const Cols x = s_o[w][lane];
#pragma unroll
      for (int e = 0; e < E; ++e) o.x[e] += x.x[e] * f;
    }
  }
  if (!live) return;
  const size_t row = (size_t)b * p.H + kvh * p.G + part * heads_unit + h;
  const float r = one_over(l);
#pragma unroll
  for (int e = 0; e < E; ++e) store_out<T>(p, row, lane * E + e, DH, o.x[e] * r);
  if (lane == 0) store_lse(p, row, m, l);
}

// How a call is cut up: heads of a unit, units of a KV head, CTAs (and of them in a cluster, 0: shares and a join).
struct PagedPlan {
  int heads_unit, units_h, ctas, min_share, joins, together;          // together: -1 a warp per unit
  bool deep;                                                             // two pages of a warp ahead, in a cluster
  long long units;
};
// A cluster per unit, as many CTAs as let all run at once and find a page for each of their warps, while the longest sequence leaves a warp no more than 12 pages;
// shares and a join beyond that.  (bf16, 4 x 8 heads of 128, all sequences alike / between half as long and as long, every fourth idle; us with
// clusters, with shares: 64 units of 8 pages 5.8 / 5.8, 7.0 / 13.0; 8 of 400 11.4 / 9.6, 13.4 / 15.2; 192 of 64 19.7 / 17.9, 23.3 / 19.5; 1 of 400 8.4, 9.8.  More than
// that to a warp, the longest decide: 256 units of 64 29.6 / 27.9, 28.2 / 21.8; 128 of 160 35.8 / 32.2, 36.4 / 24.3; 1 of 1000 14.1, 10.6.  And of more than one wave: 512 units
// of 32 35.9 / 22.8, 30.3 / 23.8; 2048 of 24 82 / 56, 73 / 52.  fp32 with eight heads to a unit, or four of 128: half as many, 32 units of 300 pages, 8 heads of 128, 34.4 / 29.7, 36.2 / 25.2;
// four heads of 64: 128 units of 60 13.7 / 12.1, 16.4 / 14.2; 400 of 40 23.8 / 15.6, 28.5 / 18.2.)
constexpr int kClusterPages = 12;
// Many short sequences: a warp per unit, while that is no more pages than these (four times as many where the units are more than one wave of CTAs).  (Pages of a sequence, all
// alike, us with a CTA / a warp per unit: 384 units of 1 / 4 / 8 pages 6.6 / 7.7 / 9.0, 4.8 / 7.1 / 9.6; 1024 of 1 / 8 / 16 18.7 / 27.0 / 36.5, 6.8 / 17.3 / 28.8; 5120 of 1 / 8
// 75 / 108, 19 / 59.)
constexpr int kWarpPages = 4;
// Groups of more than eight heads in bf16: sixteen to a unit, which reads keys and values once for them; eight, and more CTAs, while those are no more pages than these in all.  (Heads of
// 128, us with 16 / 8: 2 units of 256 pages 8.5 / 7.0, 32 of 64 14.0 / 8.4, 512 of 4 12.6 / 8.7; 32 of 256 19.9 / 17.0, ragged 11.9 / 15.6; 128 of 64 12.1 / 18.4; 512 of 256 102 / 167.)
constexpr int kFewPages = 4096;
// Shares of fewer items cost more in joins than they save.  (1 unit of 64 pages, 4 / 8 / 16 items: 7.6 / 7.8 / 9.2 us; 64 of 24: 10.9 / 10.2 / 11.6.)
// Of units that have fewer in the mean, a share takes one: else up to eight stand one behind another.  (512 units of a page, at most 512 by the caller's word, 20.9 -> 7.5 us.)
constexpr int kMinShare = 8;
// Clusters of so many CTAs that run at once, with this many CTAs to an SM: those of a cluster lie in one of the GPU's eight parts, whose SMs are no multiple of them.  One more, and the last run when
// the first have ended.  (us, units of 60 pages: 32 / 34 in clusters of 8, two to an SM, 6.7 / 10.3; 46 / 50, three to an SM, 7.6 / 11.0; 14 / 16 in clusters of 16, two to an SM, 8.7 / 15.6;
// 70 / 74 in clusters of 4, two to an SM, 8.7 / 13.6.)
constexpr int clusters_at_once(int together, int per_sm) { return per_sm * (together == 16 ? 7 : together == 8 ? 16 : together == 4 ? 35 : 148 / together); }
// max_items: pages that a sequence can have to be looked at (a window may begin and end inside one)
int plan_paged(int dtype, int B, int H, int Hk, int head_dim, int max_len, int window, int max_sel, PagedPlan* g) {
  if (dtype != CERB_F32 && dtype != CERB_BF16) return CERB_E_ARG;
  if (B < 0 || H < 1 || Hk < 1 || H % Hk || (head_dim != 64 && head_dim != 128) || max_sel > kMaxList) return CERB_E_SHAPE;
  const long long whole = ((long long)max_len + CERB_PAGE - 1) / CERB_PAGE, in_window = ((long long)window + 2 * CERB_PAGE - 2) / CERB_PAGE;
  const long long items = max_sel > 0 ? std::min((long long)max_sel, whole) : window > 0 && in_window < whole ? in_window : whole;
  const int G = H / Hk;
  const bool bf = dtype == CERB_BF16;
  g->heads_unit = bf ? (G > 8 && (long long)B * Hk * ((G + 7) / 8) * items > kFewPages ? 16 : 8) : G > 4 ? 8 : G > 2 ? 4 : G;
  g->units_h = (G + g->heads_unit - 1) / g->heads_unit;
  g->units = (long long)B * Hk * g->units_h;
  if (g->units * std::max(g->heads_unit, PA_CLUSTER) > 0x7fffffffll) return CERB_E_SHAPE;
  const int per_sm = bf ? (g->heads_unit == 8 ? ctas_per_sm<bf16, 64, 8>() : ctas_per_sm<bf16, 64, 16>())
                        : g->heads_unit == 8 ? (head_dim == 64 ? ctas_per_sm<float, 64, 8>() : ctas_per_sm<float, 128, 8>())
                        : g->heads_unit == 4 ? ctas_per_sm<float, 64, 4>() : ctas_per_sm<float, 64, 2>();
  const int at_once = 148 * per_sm;
  // (bf16, more units than seven: sixteen CTAs only where eight leave a warp many pages, us with 8 / 16: 8 units of 60 pages 5.2 / 5.6, of 200 7.9 / 8.1, of 400 11.9 / 10.7, of a list of 256 10.3 / 9.2; heads of 64, of 60
  // 4.3 / 4.6, of 120 5.6 / 5.1)
  const int widest = bf && g->units > 7 && items <= (head_dim == 64 ? 64 : 192) ? 8 : PA_CLUSTER;
  g->together = 1;
  while (g->together < widest && g->units <= clusters_at_once(2 * g->together, per_sm) && g->together * 2 * PA_WARPS <= items + PA_WARPS) g->together *= 2;
  if (g->units > at_once || items > (long long)g->together * PA_WARPS * (bf || g->heads_unit <= 2 || g->heads_unit * head_dim == 256 ? kClusterPages : kClusterPages / 2)) g->together = 0;
  g->min_share = kMinShare;
  if (g->units > at_once ? items <= 4 * kWarpPages : g->units * 2 > at_once && items <= kWarpPages) g->together = -1;
  if (g->together < 0) {
    g->ctas = (int)((g->units + PA_WARPS - 1) / PA_WARPS);
    g->joins = 0;
    return CERB_OK;
  }
  if (g->together) {
    g->ctas = (int)g->units * g->together;
    g->joins = 0;
    // while two CTAs to an SM are enough, and a warp has more than one page, the warps have the registers for two pages ahead (64 units of 32 / 64 pages 8.0 / 10.3 -> 6.6 / 8.4 us,
    // 128 of 32 / 64 10.5 / 16.7 -> 9.0 / 14.5; in shares, and with fewer CTAs to have it so: no gain)
    g->deep = bf && g->units <= clusters_at_once(g->together, 2) && items > g->together * PA_WARPS * (128 / head_dim);
    return CERB_OK;
  }
  const long long most = std::max(1ll, (g->units * items + g->min_share - 1) / g->min_share);
  g->ctas = (int)std::min((long long)at_once, most);
  g->joins = (int)std::min(g->units, (long long)g->ctas);
  return CERB_OK;
}
size_t meta_bytes(const PagedPlan& g) { return ((size_t)g.joins * sizeof(int4) + 255) & ~(size_t)255; }
size_t part_ml_bytes(const PagedPlan& g) { return ((size_t)2 * g.ctas * g.heads_unit * 2 * sizeof(float) + 255) & ~(size_t)255; }
size_t scratch_bytes(const PagedPlan& g, int head_dim) {
  return g.units && !g.together ? meta_bytes(g) + part_ml_bytes(g) + (size_t)2 * g.ctas * g.heads_unit * head_dim * sizeof(float) : 0;
}

template <typename T, int DH, int HEADS, int AHEAD>
cudaError_t launch_cluster(const PagedPlan& g, const PagedParams& p, cudaStream_t st) {
  auto kern = paged_attn_cluster_kernel<T, DH, HEADS, AHEAD>;
  if (g.together > 8) {
    static std::atomic<uint64_t> done{0};
    if (allow_wide_clusters(kern, done) != CERB_OK) return cudaErrorInvalidValue;
  }
  return launch_pdl_cluster(kern, dim3((unsigned)g.ctas), dim3(PA_WARPS * 32), 0, st, (unsigned)g.together, p);
}

template <typename T, int DH, int HEADS>
cudaError_t launch(const PagedPlan& g, const PagedParams& p, cudaStream_t st) {
  const dim3 block(PA_WARPS * 32);
  if (g.together < 0) return launch_pdl(paged_attn_warp_kernel<T, DH, HEADS>, dim3((unsigned)g.ctas), block, 0, st, p);
  if (g.together) {
    constexpr bool deep = sizeof(T) == 2 && HEADS == 8;
    return deep && g.deep ? launch_cluster<T, DH, HEADS, deep ? 2 : 1>(g, p, st) : launch_cluster<T, DH, HEADS, 1>(g, p, st);
  }
  const cudaError_t rc = launch_pdl(paged_attn_kernel<T, DH, HEADS>, dim3((unsigned)g.ctas), block, 0, st, p);
  if (rc != cudaSuccess || g.ctas == 1) return rc;
  // as many CTAs as run at once, of as many warps as there are parts to a unit
  int y = 1, groups = 1;
  while (y < HEADS && g.joins * y * 2 <= 2 * 148) y *= 2;
  const int heads_y = HEADS / y;
  while (2 * groups * heads_y <= 32 && groups * g.joins < g.ctas) groups *= 2;
  return launch_pdl(paged_join_kernel<T, DH>, dim3((unsigned)g.joins, (unsigned)y), dim3((unsigned)(32 * heads_y * groups)), 0, st, p, HEADS, heads_y);
}

}  // namespace

}  // namespace cerb

using namespace cerb;

extern "C" {

int cerb_paged_attention_scratch_bytes(int32_t dtype, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_len, int32_t window,
                                       int32_t max_sel, size_t* bytes_out) {
  if (!bytes_out || max_len < 1 || window < 0 || max_sel < 0) return CERB_E_ARG;
  PagedPlan g;
  CERB_TRY(plan_paged(dtype, B, n_heads, n_kv_heads, head_dim, max_len, window, max_sel, &g));
  *bytes_out = scratch_bytes(g, head_dim);
  return CERB_OK;
}

int cerb_paged_attention(const cerb_paged_attn_args* a, void* stream) {
  if (!a || !a->sel != !a->n_sel) return CERB_E_ARG;
  if (a->B > 0 && (!a->q || !a->k_pool || !a->v_pool || !a->page_table || !a->len || !a->out)) return CERB_E_ARG;
  if (a->max_pages < 1 || a->max_pages > (1 << 26) || a->n_pool_pages < 1 || a->max_len < 1 || a->window < 0 || (a->sel && a->max_sel < 1)) return CERB_E_ARG;
  const int max_sel = a->sel ? a->max_sel : 0;
  PagedPlan g;
  CERB_TRY(plan_paged(a->dtype, a->B, a->n_heads, a->n_kv_heads, a->head_dim, a->max_len, a->window, max_sel, &g));
  const int es = a->dtype == CERB_BF16 ? 2 : 4;
  if (a->q_row_stride * es % 16 || a->q_head_stride * es % 16) return CERB_E_ARG;
  if (((uintptr_t)a->q | (uintptr_t)a->k_pool | (uintptr_t)a->v_pool | (uintptr_t)a->out | (uintptr_t)a->scratch) & 15) return CERB_E_ARG;
  const size_t need = scratch_bytes(g, a->head_dim);
  if (need > a->scratch_bytes || (need && !a->scratch)) return CERB_E_NOMEM;
  if (a->B == 0) return CERB_OK;
  PagedParams p;
  memset(&p, 0, sizeof(p));
  p.q = a->q;
  p.k_pool = a->k_pool;
  p.v_pool = a->v_pool;
  p.page_table = a->page_table;
  p.len = a->len;
  p.sel = a->sel;
  p.n_sel = a->n_sel;
  p.out = a->out;
  p.lse = a->lse;
  p.meta = (int4*)a->scratch;
  p.by_unit = g.units <= g.ctas;
  p.part_ml = (float*)((char*)a->scratch + meta_bytes(g));
  p.part_o = (float*)((char*)p.part_ml + part_ml_bytes(g));
  p.q_row = a->q_row_stride;
  p.q_head = a->q_head_stride;
  p.B = a->B;
  p.H = a->n_heads;
  p.Hk = a->n_kv_heads;
  p.G = a->n_heads / a->n_kv_heads;
  p.units_h = g.units_h;
  p.max_pages = a->max_pages;
  p.n_pool_pages = a->n_pool_pages;
  p.max_sel = a->max_sel;
  p.window = a->window;
  p.min_share = g.min_share;
  p.together = g.together;
  p.scale_log2 = a->scale * kLog2e;
  cudaStream_t st = (cudaStream_t)stream;
  const bool wide = a->head_dim == 128;
  cudaError_t rc;
  if (a->dtype == CERB_BF16)
    rc = g.heads_unit == 16 ? (wide ? launch<bf16, 128, 16>(g, p, st) : launch<bf16, 64, 16>(g, p, st))
                            : (wide ? launch<bf16, 128, 8>(g, p, st) : launch<bf16, 64, 8>(g, p, st));
  else
    switch (g.heads_unit) {
      case 1: rc = wide ? launch<float, 128, 1>(g, p, st) : launch<float, 64, 1>(g, p, st); break;
      case 2: rc = wide ? launch<float, 128, 2>(g, p, st) : launch<float, 64, 2>(g, p, st); break;
      case 4: rc = wide ? launch<float, 128, 4>(g, p, st) : launch<float, 64, 4>(g, p, st); break;
      default: rc = wide ? launch<float, 128, 8>(g, p, st) : launch<float, 64, 8>(g, p, st);
    }
  return rc == cudaSuccess ? CERB_OK : CERB_E_CUDA;
}

}  // extern "C"
