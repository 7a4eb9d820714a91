// Attention of one new token per sequence over a paged cache whose KV heads are shared by groups of query heads, all of it or the pages of a list.
//
//   out[b][h] = sum_s softmax_s(scale q[b][h] . k[s]) v[s],  lse = ln sum_s exp(scale q . k[s]),
//   s over the slots [max(0, len - window), len), with a list over those of them that lie in its pages.
//
// Bound by HBM: every key and value once, for all query heads of its group.  A warp takes a page of 16 keys at a time, alone, from global
// memory straight into the fragments of warp MMAs: no shared memory, no barriers until the end.  The sums run as one online softmax per warp;
// the warps of a CTA meet in shared memory, the CTAs that a long cache is split over in a second kernel.
#include <math.h>
#include <string.h>

#include "cerb_internal.cuh"

namespace cerb {

namespace {

constexpr int PA_WARPS = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PagedParams {
  const void *q, *k_pool, *v_pool;
  const int32_t *page_table, *len, *sel, *n_sel;
  void* out;
  float* lse;
  float *part_o, *part_ml;        // [unit][split][heads of a unit][Dh], [..][2]
  long long q_row, q_head;        // elements
  int B, H, Hk, G, units_h;       // units_h: units per KV head (groups of more heads than a unit takes)
  int max_pages, n_pool_pages, max_sel, window;
  int nsplit, chunk;              // splits and pages of one
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
__device__ __forceinline__ int splits_of(const PagedParams& p, int items) { return min(p.nsplit, (items + p.chunk - 1) / p.chunk); }

// The page of an item: its number among the sequence's, and where it lies (-1: nothing to read there).
struct PageRef {
  int page, at;
};
__device__ __forceinline__ PageRef page_ref(const PagedParams& p, const Span& s, int b, int kvh, int item) {
  PageRef r{-1, -1};
  if (item >= s.items) return r;
  r.page = p.sel ? p.sel[((size_t)b * p.Hk + kvh) * p.max_sel + item] : s.first + item;
  if (r.page < 0 || r.page >= (s.hi + CERB_PAGE - 1) / CERB_PAGE) return r;
  const int at = p.page_table[(size_t)b * p.max_pages + r.page];
  if (at >= 0 && at < p.n_pool_pages) r.at = at;
  return r;
}

__device__ __forceinline__ uint4 ld16(const void* src) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(src) : "memory");
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}

// One CTA's part (its running maximum, sum and unnormalised outputs per head) as result or as partial.
// s_o [warp][head][DH], s_m and s_l [warp][head]
template <typename T, int DH, int HEADS>
__device__ __forceinline__ void finish_cta(const PagedParams& p, const float* s_o, const float* s_m, const float* s_l, int unit, int split, int live,
                                           int b, int head0, int heads) {
  __syncthreads();
  for (int i = threadIdx.x; i < heads * DH; i += PA_WARPS * 32) {
    const int h = i / DH, d = i % DH;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < PA_WARPS; ++w) m = fmaxf(m, s_m[w * HEADS + h]);
    const float u = m == -INFINITY ? 0.f : m;
    float l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < PA_WARPS; ++w) {
      const float f = exp2f(s_m[w * HEADS + h] - u);
      l += s_l[w * HEADS + h] * f;
      o += s_o[(w * HEADS + h) * DH + d] * f;
    }
    if (live > 1) {
      const size_t at = ((size_t)unit * p.nsplit + split) * HEADS + h;
      p.part_o[at * DH + d] = o;
      if (d == 0) { p.part_ml[2 * at] = m; p.part_ml[2 * at + 1] = l; }
    } else {
      const size_t row = (size_t)b * p.H + head0 + h;
      const float x = l > 0.f || l != l ? o / l : 0.f;                   // (a row without keys: zeros)
      if constexpr (sizeof(T) == 2) reinterpret_cast<bf16*>(p.out)[row * DH + d] = __float2bfloat16_rn(x);
      else reinterpret_cast<float*>(p.out)[row * DH + d] = x;
      if (d == 0 && p.lse) p.lse[row] = (m + log2f(l)) * kLn2;
    }
  }
}

// bf16.  Both products have the keys (of K q: 16 keys; of V p: Dh) on the MMA's 16 rows and the heads, NT groups of eight, on its columns: S^T = K q^T,
// out^T = V^T P^T.  The order of the k positions of a product is free as long as both operands have the same, so a lane's 16
// bytes of a key row (8 consecutive elements) are what it needs of two MMAs, and what it loads of the values, 8 elements of each of four keys, is
// interleaved into fragments by byte permutes.  S^T's sums become P^T's fragments by two 8 x 8 transpositions of 16-bit elements.
// P is rounded to bf16 for the second product (each weight off by at most 2^-9 of itself, in turns up and down; the sum l is that of the unrounded
// ones); scores, maxima, sums and outputs are fp32.
template <int DH, int NT>
__global__ void __launch_bounds__(PA_WARPS * 32, NT == 1 ? 4 : 2) paged_attn_bf16_kernel(const PagedParams p) {
  constexpr int HEADS = 8 * NT, KC = DH / 32, VH = DH / 64;              // chunks of a key row, halves of a value row
  __shared__ float s_o[PA_WARPS * HEADS * DH];
  __shared__ float s_m[PA_WARPS * HEADS], s_l[PA_WARPS * HEADS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x % p.nsplit, unit = blockIdx.x / p.nsplit;
  const int part = unit % p.units_h, kvh = unit / p.units_h % p.Hk, b = unit / p.units_h / p.Hk;
  griddep_wait();
  griddep_launch();
  const Span sp = span_of(p, b);
  const int live = splits_of(p, sp.items);
  if (split >= max(live, 1)) return;
  const int head0 = kvh * p.G + part * HEADS, heads = min(HEADS, p.G - part * HEADS);
  const bf16* kp = reinterpret_cast<const bf16*>(p.k_pool) + (size_t)kvh * CERB_PAGE * DH + g * DH + t * 8;
  const bf16* vp = reinterpret_cast<const bf16*>(p.v_pool) + (size_t)kvh * CERB_PAGE * DH + 2 * t * DH + g * 8;
  const size_t page_elems = (size_t)p.Hk * CERB_PAGE * DH;
  uint4 q[NT][KC];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < KC; ++j)
      q[n][j] = 8 * n + g < heads
                    ? *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(p.q) + (size_t)b * p.q_row + (size_t)(head0 + 8 * n + g) * p.q_head + 32 * j + 8 * t)
                    : make_uint4(0, 0, 0, 0);
  uint4 k[2][KC], v[4][VH];
  auto load_k = [&](int at) {
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < KC; ++j) k[r][j] = ld16(kp + at * page_elems + r * 8 * DH + 32 * j);
  };
  auto load_v = [&](int at) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < VH; ++j) v[r][j] = ld16(vp + at * page_elems + ((r & 1) + 8 * (r >> 1)) * DH + 64 * j);
  };
  float o[NT][4 * VH][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n][0] = m[n][1] = -INFINITY;
    l[n][0] = l[n][1] = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * VH; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
  }
  // this warp's items: every PA_WARPS-th of a split's chunk, and of those nsplit chunks on (none, unless a sequence is longer than the caller said)
  const int per = p.chunk / PA_WARPS;                                    // (chunk is a multiple of PA_WARPS)
  auto item_of = [&](int i) { return (split + i / per * p.nsplit) * p.chunk + i % per * PA_WARPS + warp; };
  int i = 0, pages_l = -1, at_l = -1;
  PageRef now{-1, -1};
  // the next item that there is something to read of, or -1
  auto next = [&]() {
    PageRef r{-1, -1};
    for (;;) {
      if (item_of(i) >= sp.items) break;                                 // (items only grow)
      if (i % 32 == 0) {
        const PageRef mine = page_ref(p, sp, b, kvh, item_of(i + lane));
        pages_l = mine.page;
        at_l = mine.at;
      }
      r.page = __shfl_sync(0xffffffffu, pages_l, i % 32);
      r.at = __shfl_sync(0xffffffffu, at_l, i % 32);
      ++i;
      if (r.at >= 0) break;
    }
    return r;
  };
  now = next();
  if (now.at >= 0) { load_k(now.at); load_v(now.at); }
  while (now.at >= 0) {
    const PageRef then = next();
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      // (two accumulators: the tensor cores cut a sum off at every step)
      float a0[4] = {0.f, 0.f, 0.f, 0.f}, a1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        mma_16816(a0, k[0][j].x, k[1][j].x, k[0][j].y, k[1][j].y, q[n][j].x, q[n][j].y);
        mma_16816(a1, k[0][j].z, k[1][j].z, k[0][j].w, k[1][j].w, q[n][j].z, q[n][j].w);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = (a0[e] + a1[e]) * p.scale_log2;
    }
    if (then.at >= 0) load_k(then.at);
    const int row0 = now.page * CERB_PAGE;
    if (row0 < sp.lo || row0 + CERB_PAGE > sp.hi) {
      // the ends: whatever lies outside counts nothing, and is nothing (it may be infinite)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = row0 + g + 8 * (e >> 1);
          if (r < sp.lo || r >= sp.hi) s[n][e] = -INFINITY;
        }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = row0 + 2 * t + (r & 1) + 8 * (r >> 1);
        if (row < sp.lo || row >= sp.hi)
#pragma unroll
          for (int j = 0; j < VH; ++j) v[r][j] = make_uint4(0, 0, 0, 0);
      }
    }
    uint32_t pb[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float mx[2] = {fmaxf(s[n][0], s[n][2]), fmaxf(s[n][1], s[n][3])};
#pragma unroll
      for (int w = 4; w < 32; w <<= 1)
#pragma unroll
        for (int e = 0; e < 2; ++e) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], w));
      float a[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mx[e] = fmaxf(mx[e], m[n][e]);
        const float u = mx[e] == -INFINITY ? 0.f : mx[e];
        a[e] = exp2f(m[n][e] - u);
        m[n][e] = mx[e];
        s[n][e] = exp2f(s[n][e] - u);
        s[n][e + 2] = exp2f(s[n][e + 2] - u);
        l[n][e] = l[n][e] * a[e] + s[n][e] + s[n][e + 2];
      }
      if (__any_sync(0xffffffffu, a[0] != 1.f || a[1] != 1.f)) {
#pragma unroll
        for (int c = 0; c < 4 * VH; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[n][c][e] *= a[e & 1];
      }
      pb[n][0] = transpose8x8(pack_bf16(s[n][0], s[n][1]));
      pb[n][1] = transpose8x8(pack_bf16(s[n][2], s[n][3]));
    }
#pragma unroll
    for (int j = 0; j < VH; ++j) {
      const uint32_t x[4][4] = {{v[0][j].x, v[0][j].y, v[0][j].z, v[0][j].w}, {v[1][j].x, v[1][j].y, v[1][j].z, v[1][j].w},
                                {v[2][j].x, v[2][j].y, v[2][j].z, v[2][j].w}, {v[3][j].x, v[3][j].y, v[3][j].z, v[3][j].w}};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t a0 = __byte_perm(x[0][c], x[1][c], 0x5410), a1 = __byte_perm(x[0][c], x[1][c], 0x7632);
        const uint32_t a2 = __byte_perm(x[2][c], x[3][c], 0x5410), a3 = __byte_perm(x[2][c], x[3][c], 0x7632);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_16816(o[n][4 * j + c], a0, a1, a2, a3, pb[n][0], pb[n][1]);
      }
    }
    if (then.at >= 0) load_v(then.at);
    now = then;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], w);
      const int h = warp * HEADS + 8 * n + 2 * t + e;
      if (g == 0) { s_m[h] = m[n][e]; s_l[h] = l[n][e]; }
      // accumulator c of half j: rows g and g + 8 of the MMA are the elements 2c and 2c + 1 of the lane's eight
#pragma unroll
      for (int c = 0; c < 4 * VH; ++c)
        *reinterpret_cast<float2*>(&s_o[h * DH + (c >> 2) * 64 + 8 * g + 2 * (c & 3)]) = make_float2(o[n][c][e], o[n][c][e + 2]);
    }
  finish_cta<bf16, DH, HEADS>(p, s_o, s_m, s_l, unit, split, live, b, head0, heads);
}

// fp32: plain FMA.  A lane owns DH / 32 elements of every key and value, a warp takes eight keys at a time for up to GH heads.  The lanes' 8 GH partial sums
// meet by halving (every exchange carries half of what is left: as many shuffles as sums), after which each lane has the scores of few keys to
// take the exponential of; the weights come back by shuffles.
template <int N>
__device__ __forceinline__ void halve_sums(float (&x)[N], int lane) {
  int n = N;
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) {
    if (n > 1) {
      n >>= 1;
      const bool up = lane & w;
#pragma unroll
      for (int i = 0; i < N / 2; ++i)
        if (i < n) {
          const float send = up ? x[i] : x[i + n], keep = up ? x[i + n] : x[i];
          x[i] = keep + __shfl_xor_sync(0xffffffffu, send, w);
        }
    } else {
      x[0] += __shfl_xor_sync(0xffffffffu, x[0], w);
    }
  }
}

template <int DH, int GH>
__global__ void __launch_bounds__(PA_WARPS * 32) paged_attn_f32_kernel(const PagedParams p) {
  constexpr int E = DH / 32, NV = 8 * GH, R = NV >= 32 ? NV / 32 : 1, REP = NV >= 32 ? 1 : 32 / NV, LPH = 32 / GH;       // sums of a lane at the end, lanes with the same one; lanes of a head
  __shared__ float s_o[PA_WARPS * GH * DH];
  __shared__ float s_m[PA_WARPS * GH], s_l[PA_WARPS * GH];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = blockIdx.x % p.nsplit, unit = blockIdx.x / p.nsplit;
  const int part = unit % p.units_h, kvh = unit / p.units_h % p.Hk, b = unit / p.units_h / p.Hk;
  griddep_wait();
  griddep_launch();
  const Span sp = span_of(p, b);
  const int live = splits_of(p, sp.items);
  if (split >= max(live, 1)) return;
  const int head0 = kvh * p.G + part * GH, heads = min(GH, p.G - part * GH);
  const size_t page_elems = (size_t)p.Hk * CERB_PAGE * DH;
  const float* kp = reinterpret_cast<const float*>(p.k_pool) + (size_t)kvh * CERB_PAGE * DH + lane * E;
  const float* vp = reinterpret_cast<const float*>(p.v_pool) + (size_t)kvh * CERB_PAGE * DH + lane * E;
  struct Row {
    float x[E];
  };
  auto load_row = [](const float* src) {
    Row r;
    if constexpr (E == 4)
      asm volatile("ld.global.L1::no_allocate.L2::256B.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(r.x[0]), "=f"(r.x[1]), "=f"(r.x[2]), "=f"(r.x[3]) : "l"(src) : "memory");
    else
      asm volatile("ld.global.L1::no_allocate.L2::256B.v2.f32 {%0, %1}, [%2];" : "=f"(r.x[0]), "=f"(r.x[1]) : "l"(src) : "memory");
    return r;
  };
  float q[GH][E], o[GH][E];
#pragma unroll
  for (int h = 0; h < GH; ++h)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[h][e] = h < heads ? reinterpret_cast<const float*>(p.q)[(size_t)b * p.q_row + (size_t)(head0 + h) * p.q_head + lane * E + e] : 0.f;
      o[h][e] = 0.f;
    }
  float m = -INFINITY, l = 0.f;                                          // of head lane / LPH
  const int per = p.chunk / PA_WARPS;
  for (int i = 0;; ++i) {
    const int item = (split + i / per * p.nsplit) * p.chunk + i % per * PA_WARPS + warp;
    if (item >= sp.items) break;
    const PageRef r = page_ref(p, sp, b, kvh, item);
    if (r.at < 0) continue;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int row0 = r.page * CERB_PAGE + half * 8;
      if (row0 >= sp.hi || row0 + 8 <= sp.lo) continue;
      Row k[8], v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) k[j] = load_row(kp + r.at * page_elems + (half * 8 + j) * DH);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = load_row(vp + r.at * page_elems + (half * 8 + j) * DH);
      float s[NV];                                                       // [head][key]
#pragma unroll
      for (int h = 0; h < GH; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float x = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) x = fmaf(q[h][e], k[j].x[e], x);
          s[h * 8 + j] = x;
        }
      halve_sums(s, lane);
      float mx = m;
      const bool ends = row0 < sp.lo || row0 + 8 > sp.hi;
#pragma unroll
      for (int c = 0; c < R; ++c) {
        s[c] *= p.scale_log2;
        const int row = row0 + (lane / REP * R + c) % 8;
        if (ends && (row < sp.lo || row >= sp.hi)) s[c] = -INFINITY;
        mx = fmaxf(mx, s[c]);
      }
      if (ends) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (row0 + j < sp.lo || row0 + j >= sp.hi)
#pragma unroll
            for (int e = 0; e < E; ++e) v[j].x[e] = 0.f;
      }
#pragma unroll
      for (int w = 1; w < LPH; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float u = mx == -INFINITY ? 0.f : mx, a = exp2f(m - u);
      m = mx;
      l *= a;
#pragma unroll
      for (int c = 0; c < R; ++c) {
        s[c] = exp2f(s[c] - u);
        if (lane % REP == 0) l += s[c];
      }
#pragma unroll
      for (int h = 0; h < GH; ++h) {
        const float ah = __shfl_sync(0xffffffffu, a, h * LPH);
#pragma unroll
        for (int e = 0; e < E; ++e) o[h][e] *= ah;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int idx = h * 8 + j;
          const float w = __shfl_sync(0xffffffffu, s[idx % R], idx / R * REP);
#pragma unroll
          for (int e = 0; e < E; ++e) o[h][e] = fmaf(w, v[j].x[e], o[h][e]);
        }
      }
    }
  }
#pragma unroll
  for (int w = 1; w < LPH; w <<= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
  if (lane % LPH == 0) { s_m[warp * GH + lane / LPH] = m; s_l[warp * GH + lane / LPH] = l; }
#pragma unroll
  for (int h = 0; h < GH; ++h)
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[(warp * GH + h) * DH + lane * E + e] = o[h][e];
  finish_cta<float, DH, GH>(p, s_o, s_m, s_l, unit, split, live, b, head0, heads);
}

// The splits of a unit as one, a head per CTA and a column per thread.
template <typename T, int DH>
__global__ void __launch_bounds__(DH) paged_join_kernel(const PagedParams p, int heads_unit) {
  const int unit = blockIdx.x / heads_unit, h = blockIdx.x % heads_unit, d = threadIdx.x;
  const int part = unit % p.units_h, kvh = unit / p.units_h % p.Hk, b = unit / p.units_h / p.Hk;
  griddep_wait();
  griddep_launch();
  const int live = splits_of(p, span_of(p, b).items);
  if (live <= 1 || part * heads_unit + h >= p.G) return;
  const size_t at0 = (size_t)unit * p.nsplit * heads_unit + h;
  float m = -INFINITY;
  for (int s = 0; s < live; ++s) m = fmaxf(m, p.part_ml[2 * (at0 + (size_t)s * heads_unit)]);
  const float u = m == -INFINITY ? 0.f : m;
  float l = 0.f, o = 0.f;
#pragma unroll 4
  for (int s = 0; s < live; ++s) {
    const size_t at = at0 + (size_t)s * heads_unit;
    const float f = exp2f(p.part_ml[2 * at] - u);
    l += p.part_ml[2 * at + 1] * f;
    o += p.part_o[at * DH + d] * f;
  }
  const size_t row = (size_t)b * p.H + kvh * p.G + part * heads_unit + h;
  const float x = l > 0.f || l != l ? o / l : 0.f;
  if constexpr (sizeof(T) == 2) reinterpret_cast<bf16*>(p.out)[row * DH + d] = __float2bfloat16_rn(x);
  else reinterpret_cast<float*>(p.out)[row * DH + d] = x;
  if (d == 0 && p.lse) p.lse[row] = (m + log2f(l)) * kLn2;
}

// How a call is cut up: heads of a unit, units of a KV head, splits and the pages of one.
struct PagedPlan {
  int heads_unit, units_h, nsplit, chunk;
  long long units;
};
int plan_paged(int dtype, int B, int H, int Hk, int head_dim, int max_items, PagedPlan* g) {
  if (dtype != CERB_F32 && dtype != CERB_BF16) return CERB_E_ARG;
  if (B < 0 || H < 1 || Hk < 1 || H % Hk || (head_dim != 64 && head_dim != 128) || max_items < 1) return CERB_E_SHAPE;
  const int G = H / Hk;
  g->heads_unit = dtype == CERB_BF16 ? (G > 8 ? 16 : 8) : G > 4 ? 8 : G > 2 ? 4 : G;
  g->units_h = (G + g->heads_unit - 1) / g->heads_unit;
  g->units = (long long)B * Hk * g->units_h;
  // splits: enough CTAs for every SM several times over, of no less than 16 pages
  long long want = g->units ? (148 * 16 + g->units - 1) / g->units : 1;
  int chunk = (int)((max_items + want - 1) / want);
  chunk = (chunk + PA_WARPS - 1) / PA_WARPS * PA_WARPS;
  if (chunk < 16) chunk = 16;
  g->chunk = chunk;
  g->nsplit = (max_items + chunk - 1) / chunk;
  if (g->units * g->nsplit > 0x7fffffffll || g->units * g->heads_unit > 0x7fffffffll) return CERB_E_SHAPE;
  return CERB_OK;
}
// Pages that a sequence can have to be looked at: a window may begin and end inside one.
int max_items(int max_len, int window, int max_sel) {
  if (max_sel > 0) return max_sel;
  const int whole = (int)(((long long)max_len + CERB_PAGE - 1) / CERB_PAGE);
  const long long part = ((long long)window + 2 * CERB_PAGE - 2) / CERB_PAGE;
  return window > 0 && part < whole ? (int)part : whole;
}
size_t part_ml_bytes(const PagedPlan& g) { return ((size_t)g.units * g.nsplit * g.heads_unit * 2 * sizeof(float) + 255) & ~(size_t)255; }

}  // namespace

}  // namespace cerb

using namespace cerb;

extern "C" {

int cerb_paged_attention_scratch_bytes(int32_t dtype, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_len, int32_t window,
                                       int32_t max_sel, size_t* bytes_out) {
  if (!bytes_out || max_len < 1 || window < 0 || max_sel < 0) return CERB_E_ARG;
  PagedPlan g;
  CERB_TRY(plan_paged(dtype, B, n_heads, n_kv_heads, head_dim, max_items(max_len, window, max_sel), &g));
  *bytes_out = g.nsplit > 1 ? part_ml_bytes(g) + (size_t)g.units * g.nsplit * g.heads_unit * head_dim * sizeof(float) : 0;
  return CERB_OK;
}

int cerb_paged_attention(const cerb_paged_attn_args* a, void* stream) {
  if (!a || !a->sel != !a->n_sel) return CERB_E_ARG;
  if (a->B > 0 && (!a->q || !a->k_pool || !a->v_pool || !a->page_table || !a->len || !a->out)) return CERB_E_ARG;
  if (a->max_pages < 1 || a->max_pages > (1 << 26) || a->n_pool_pages < 1 || a->max_len < 1 || a->window < 0 || (a->sel && a->max_sel < 1)) return CERB_E_ARG;
  const int max_sel = a->sel ? a->max_sel : 0;
  PagedPlan g;
  CERB_TRY(plan_paged(a->dtype, a->B, a->n_heads, a->n_kv_heads, a->head_dim, max_items(a->max_len, a->window, max_sel), &g));
  const int es = a->dtype == CERB_BF16 ? 2 : 4;
  if (a->q_row_stride * es % 16 || a->q_head_stride * es % 16) return CERB_E_ARG;
  if (((uintptr_t)a->q | (uintptr_t)a->k_pool | (uintptr_t)a->v_pool | (uintptr_t)a->scratch) & 15) return CERB_E_ARG;
  size_t need = 0;
  CERB_TRY(cerb_paged_attention_scratch_bytes(a->dtype, a->B, a->n_heads, a->n_kv_heads, a->head_dim, a->max_len, a->window, max_sel, &need));
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
  p.part_ml = (float*)a->scratch;
  p.part_o = (float*)((char*)a->scratch + part_ml_bytes(g));
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
  p.nsplit = g.nsplit;
  p.chunk = g.chunk;
  p.scale_log2 = a->scale * kLog2e;
  cudaStream_t st = (cudaStream_t)stream;
  void (*kern)(const PagedParams);
  const bool wide = a->head_dim == 128;
  if (a->dtype == CERB_BF16)
    kern = g.heads_unit == 16 ? (wide ? paged_attn_bf16_kernel<128, 2> : paged_attn_bf16_kernel<64, 2>)
                              : (wide ? paged_attn_bf16_kernel<128, 1> : paged_attn_bf16_kernel<64, 1>);
  else
    switch (g.heads_unit) {
      case 1: kern = wide ? paged_attn_f32_kernel<128, 1> : paged_attn_f32_kernel<64, 1>; break;
      case 2: kern = wide ? paged_attn_f32_kernel<128, 2> : paged_attn_f32_kernel<64, 2>; break;
      case 4: kern = wide ? paged_attn_f32_kernel<128, 4> : paged_attn_f32_kernel<64, 4>; break;
      default: kern = wide ? paged_attn_f32_kernel<128, 8> : paged_attn_f32_kernel<64, 8>;
    }
  if (launch_pdl(kern, dim3((unsigned)(g.units * g.nsplit)), dim3(PA_WARPS * 32), 0, st, p) != cudaSuccess) return CERB_E_CUDA;
  if (g.nsplit == 1) return CERB_OK;
  const dim3 grid((unsigned)(g.units * g.heads_unit)), block((unsigned)a->head_dim);
  cudaError_t rc;
  if (a->dtype == CERB_BF16) rc = launch_pdl(wide ? paged_join_kernel<bf16, 128> : paged_join_kernel<bf16, 64>, grid, block, 0, st, p, g.heads_unit);
  else rc = launch_pdl(wide ? paged_join_kernel<float, 128> : paged_join_kernel<float, 64>, grid, block, 0, st, p, g.heads_unit);
  return rc == cudaSuccess ? CERB_OK : CERB_E_CUDA;
}

}  // extern "C"
