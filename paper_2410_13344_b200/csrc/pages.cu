// Bookkeeping of a paged KV cache, and the append into it.
//
// Tree attention reads lengths, page tables and committed keys ahead of its wait for the kernel in front.  So the kernels here, which write them, do not
// let the next kernel start before they are complete.
#include <string.h>

#include <algorithm>

#include "cerb_internal.cuh"

namespace cerb {

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_FEW = 256;
constexpr int TRIM_CLUSTER = 8, TRIM_WIDE = 16;      // CTAs of a trim's cluster, of more requests than a CTA has threads
// Up to this many rows one CTA fills them; more are spread over the SMs, and a second launch changes the state.
// (64 requests of a token each: plan and trim 6.0 us; 300 requests, 11000 rows: 9.3; 2000 requests, a million rows, 45000 pages back: 20.5.)
constexpr int kPlanRowsAlone = 2048;
constexpr int kMaxRequests = 8192;      // four words each of a CTA's shared memory

struct PagesParams {
  int32_t *len, *page_table, *free_pages, *n_free;
  const int32_t* n_new;                 // plan: tokens that each request wants; trim: the lengths to keep
  int32_t *slot, *pos, *seq, *row_off, *granted;
  int B, max_pages, free_cap, rows;
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

__device__ __forceinline__ int pages_of(int tokens) { return (int)(((unsigned)tokens + CERB_PAGE - 1) / CERB_PAGE); }

// What a table or the stack may name as a page: those of a pool of less than 2^27 of them.
__device__ __forceinline__ bool can_be_page(int page) { return (unsigned)page < 1u << 27; }

// A slot of what a table or the stack names as a page.  (What can be no page, of a pool of less than 2^27 of them, gives a slot that nothing is written to.)
__device__ __forceinline__ int slot_of(int page, int row) { return page >= 1 << 27 ? -1 : max(page, -(1 << 27)) * CERB_PAGE + row; }

// Rows and pages, summed up together.
struct Sums {
  long long rows;
  int pages;
};
__device__ __forceinline__ Sums operator+(Sums a, Sums b) { return Sums{a.rows + b.rows, a.pages + b.pages}; }
__device__ __forceinline__ Sums shuffle_up(Sums v, int o) { return Sums{__shfl_up_sync(0xffffffffu, v.rows, o), __shfl_up_sync(0xffffffffu, v.pages, o)}; }
__device__ __forceinline__ Sums shuffle(Sums v, int i) { return Sums{__shfl_sync(0xffffffffu, v.rows, i), __shfl_sync(0xffffffffu, v.pages, i)}; }
__device__ __forceinline__ int shuffle_up(int v, int o) { return __shfl_up_sync(0xffffffffu, v, o); }
__device__ __forceinline__ int shuffle(int v, int i) { return __shfl_sync(0xffffffffu, v, i); }

// Inclusive sum over the CTA's threads; `total` is that of all.
template <int THREADS, typename T>
__device__ __forceinline__ T block_scan(T v, T* red, T& total) {
  constexpr int WARPS = THREADS / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T u = shuffle_up(v, o);
    if (lane >= o) v = v + u;
  }
  if (lane == 31) red[warp] = v;
  __syncthreads();
  T w = lane < WARPS ? red[lane] : T{};
#pragma unroll
  for (int o = 1; o < WARPS; o <<= 1) {
    const T u = shuffle_up(w, o);
    if (lane >= o) w = w + u;
  }
  total = shuffle(w, WARPS - 1);
  const T before = shuffle(w, (warp + 31) & 31);
  __syncthreads();
  return warp ? v + before : v;
}

// The lengths of a request as the kernels use them: what is out of range is taken to the nearest that is in range.
__device__ __forceinline__ int held_tokens(const PagesParams& p, int b) { return min(max(p.len[b], 0), p.max_pages * CERB_PAGE); }

// The request that item i is of, ends[b] being the first item behind request b (all lanes of a warp, one item): thirty-two bounds at a time.
__device__ __forceinline__ int find_request(const int* ends, int B, int i) {
  const int lane = threadIdx.x & 31;
  int lo = 0;
  for (int n = B; n > 1;) {
    const int step = (n + 31) / 32, at = lo + (lane + 1) * step - 1;
    const int before = __popc(__ballot_sync(0xffffffffu, at < B && at < lo + n && ends[at] <= i));
    lo += before * step;
    n = min(step, B - lo);
  }
  return min(lo, B - 1);
}
// ... and that of item i, which is of request b or of one of the next 128 with items.  (By a lane.)
__device__ __forceinline__ int find_near(const int* ends, int B, int b, int i) {
  int hi = B - 1;
  while (b < hi) {
    const int mid = (b + hi) >> 1;
    if (ends[mid] <= i) b = mid + 1;
    else hi = mid;
  }
  return b;
}

// Prefix sums over the requests (rows, and pages of those that fit) and then a row per element: its request, position and slot.
// New pages never lie where a row of this call finds an old one, so the table may change at once.  Lengths and free count change when all have read them:
// with one CTA (ALONE) at its end, with more (each of which sums up for itself) in a launch of their own.
template <int THREADS, bool ALONE>
__global__ void __launch_bounds__(THREADS, 1) pages_plan_kernel(const PagesParams p) {
  extern __shared__ __align__(16) int sm[];
  int *ends = sm, *lens = ends + p.B, *base = lens + p.B, *give = base + p.B;     // rows before and of b, length, new pages before, 1 if granted
  __shared__ Sums red[32];
  __shared__ int s_taken;
  const int tid = threadIdx.x, lane = tid & 31;
  const unsigned cta = ALONE ? 0 : blockIdx.x, ctas = ALONE ? 1 : gridDim.x;
  if (tid == 0) s_taken = 0;
  griddep_wait();
  const int n_free = min(max(*p.n_free, 0), p.free_cap);
  Sums before{0, 0};
  for (int b0 = 0; b0 < p.B; b0 += THREADS) {
    const int b = b0 + tid;
    const bool live = b < p.B;
    const int len = live ? held_tokens(p, b) : 0, n = live ? max(p.n_new[b], 0) : 0;
    // (those that do not fit the rows come last: whatever they add to the pages is added to nobody's)
    bool fits = live && (long long)len + n <= (long long)p.max_pages * CERB_PAGE;
    const int need = fits ? pages_of(len + n) - pages_of(len) : 0;
    Sums total;
    const Sums end = before + block_scan<THREADS>(Sums{n, need}, red, total);
    fits = fits && end.rows <= p.rows;
    const bool ok = fits && (need == 0 || end.pages <= n_free);
    if (live) {
      ends[b] = (int)min(end.rows, 0x7fffffffll);
      lens[b] = len;
      base[b] = end.pages - need;
      give[b] = ok;
      if (cta == 0) {
        p.granted[b] = ok ? n : 0;
        p.row_off[b + 1] = (int)min(end.rows, 0x7fffffffll);
        // (the ones with new pages that get them are the first ones)
        if (ALONE && ok && need) atomicMax(&s_taken, end.pages);
      }
    }
    before = before + total;
  }
  if (cta == 0 && tid == 0) p.row_off[0] = 0;
  __syncthreads();
  const int total = (int)min(before.rows, (long long)p.rows);
  // where page j of request b comes from
  auto source = [&](int b, int j) {
    const int held = pages_of(lens[b]);
    return j < held ? p.page_table + (size_t)b * p.max_pages + j : p.free_pages + (n_free - 1 - base[b] - (j - held));
  };
  if (ALONE || p.rows <= (int)(ctas * THREADS)) {
    // a row to a lane: with few rows the time is that of the loads one after another
    for (int r = (int)(cta * THREADS) + tid; r < p.rows; r += (int)(ctas * THREADS)) {
      int slot = -1, pos = -1, seq = -1;
      if (r < total) {
        const int b = find_near(ends, p.B, 0, r);
        if (give[b]) {
          seq = b;
          pos = lens[b] + r - (b ? ends[b - 1] : 0);
          const int j = pos / CERB_PAGE, page = *source(b, j);
          if (pos % CERB_PAGE == 0) p.page_table[(size_t)b * p.max_pages + j] = page;      // (a page that begins here is new)
          slot = slot_of(page, pos % CERB_PAGE);
        }
      }
      p.slot[r] = slot;
      p.pos[r] = pos;
      p.seq[r] = seq;
    }
  } else {
    // four rows to a lane, mostly of one request
    const bool wide = !(((uintptr_t)p.slot | (uintptr_t)p.pos | (uintptr_t)p.seq) & 15);
    for (int w0 = 4 * (int)(cta * THREADS + (tid & ~31)); w0 < p.rows; w0 += 4 * (int)(ctas * THREADS)) {
      const int r0 = w0 + 4 * lane;
      int slot[4], pos[4], seq[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) slot[i] = pos[i] = seq[i] = -1;
      int b = w0 < total ? find_request(ends, p.B, w0) : 0;
      const bool one = w0 + 127 < total && ends[b] > w0 + 127;
      if (!one && r0 < total) b = find_near(ends, p.B, b, r0);
      if (one || (r0 + 3 < total && ends[b] > r0 + 3)) {
        if (give[b]) {
          const int at = lens[b] + r0 - (b ? ends[b - 1] : 0), j = at / CERB_PAGE;
          const bool cross = (at + 3) / CERB_PAGE != j;
          const int32_t* from = source(b, j);
          const int32_t* from2 = cross ? source(b, j + 1) : from;
          const int page = *from, page2 = *from2;
          if (at % CERB_PAGE == 0 || cross) p.page_table[(size_t)b * p.max_pages + j + cross] = page2;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pos[i] = at + i;
            seq[i] = b;
            slot[i] = slot_of((at + i) / CERB_PAGE == j ? page : page2, (at + i) % CERB_PAGE);
          }
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < 4 && r0 + i < total; ++i) {
          while (ends[b] <= r0 + i) ++b;
          if (!give[b]) continue;
          const int at = lens[b] + r0 + i - (b ? ends[b - 1] : 0), page = *source(b, at / CERB_PAGE);
          if (at % CERB_PAGE == 0) p.page_table[(size_t)b * p.max_pages + at / CERB_PAGE] = page;
          const int x = slot_of(page, at % CERB_PAGE);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (k == i) { slot[k] = x; pos[k] = at; seq[k] = b; }
        }
      }
      if (wide && r0 + 3 < p.rows) {
        *reinterpret_cast<int4*>(p.slot + r0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
        *reinterpret_cast<int4*>(p.pos + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        *reinterpret_cast<int4*>(p.seq + r0) = make_int4(seq[0], seq[1], seq[2], seq[3]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (r0 + i < p.rows) { p.slot[r0 + i] = slot[i]; p.pos[r0 + i] = pos[i]; p.seq[r0 + i] = seq[i]; }
      }
    }
  }
  if (!ALONE) return;
  for (int b = tid; b < p.B; b += THREADS) {
    const int n = ends[b] - (b ? ends[b - 1] : 0);
    if (give[b] && n) p.len[b] = lens[b] + n;
  }
  if (tid == 0) *p.n_free = n_free - s_taken;
}

__global__ void __launch_bounds__(PLAN_THREADS, 1) pages_grant_kernel(const PagesParams p) {
  __shared__ int red_pages[32];
  griddep_wait();
  int taken = 0;
  for (int b = threadIdx.x; b < p.B; b += PLAN_THREADS) {
    const int n = p.granted[b], len = held_tokens(p, b);
    taken += pages_of(len + n) - pages_of(len);
    if (n) p.len[b] = len + n;
  }
  int total;
  block_scan<PLAN_THREADS>(taken, red_pages, total);
  if (threadIdx.x == 0) *p.n_free = min(max(*p.n_free, 0), p.free_cap) - total;
}

// Pages behind the lengths to keep go back to the list, the last one of the last request first: a trim to the lengths before a
// plan leaves the list as it was.  One cluster: lengths and free count change behind its barrier.
// Table entries that can be no page (of a window's old pages, say, which were given back by hand) are passed over.  They are found as the pages are written, and then the first CTA closes the gaps that
// they have left; where the stack may not have room for all, it goes through the entries by itself.  (Trim and plan of 64 requests 5.9 us without looking for them, 6.0 with; of 2000, 45000 entries,
// 19.7 and 20.5, another barrier of the cluster; counting them before anything is written 6.7 and 21.2.  With gaps: 4000 entries 6.7 us instead of 3.9, 44000 36 instead of 8, and 74 without room.)
__global__ void __launch_bounds__(PLAN_THREADS, 1) pages_trim_kernel(const PagesParams p) {
  extern __shared__ __align__(16) int sm[];
  int *ends = sm, *news = ends + p.B;                          // pages given back before and of b; the length kept
  __shared__ int red_pages[32], s_some;
  const int tid = threadIdx.x;
  const unsigned cta = blockIdx.x, ctas = gridDim.x;                 // (one cluster)
  if (tid == 0) s_some = 0;
  griddep_wait();
  const int n_free = min(max(*p.n_free, 0), p.free_cap);
  int total = 0;
  for (int b0 = 0; b0 < p.B; b0 += PLAN_THREADS) {
    const int b = b0 + tid;
    const int len = b < p.B ? held_tokens(p, b) : 0, keep = b < p.B ? min(max(p.n_new[b], 0), len) : 0;
    int t;
    const int end = total + block_scan<PLAN_THREADS>(pages_of(len) - pages_of(keep), red_pages, t);
    if (b < p.B) { ends[b] = end; news[b] = keep; }
    total += t;
  }
  cluster_arrive();
  __syncthreads();
  const bool room = (unsigned)n_free + (unsigned)total <= (unsigned)p.free_cap;
  bool some = !room;                                                     // (which of them fit, if any are no page, is seen one after another)
  // two pages to a lane  (counted in 32 bits without a sign: up to 2^31 of them, and a step past the last)
  for (unsigned w0 = 2 * (cta * PLAN_THREADS + (tid & ~31)); room && w0 < (unsigned)total; w0 += 2 * ctas * PLAN_THREADS) {
    int b = find_request(ends, p.B, (int)w0), page[2];
    int32_t* entry[2] = {nullptr, nullptr};
    const bool one = (unsigned)ends[b] > w0 + 63;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned at = w0 + 32 * i + (tid & 31);
      if (at >= (unsigned)total) continue;
      const int c = one ? b : find_near(ends, p.B, b, (int)at);
      entry[i] = p.page_table + (size_t)c * p.max_pages + pages_of(news[c]) + ((int)at - (c ? ends[c - 1] : 0));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (entry[i]) page[i] = *entry[i];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (entry[i]) {
        some |= !can_be_page(page[i]);
        p.free_pages[(unsigned)n_free + (unsigned)total - 1 - (w0 + 32 * i + (tid & 31))] = page[i];
        *entry[i] = -1;
      }
  }
  some = __syncthreads_or(some);
  cluster_wait();
  for (int b = tid; cta == 0 && b < p.B; b += PLAN_THREADS) p.len[b] = news[b];
  if ((unsigned)total > 2 * PLAN_THREADS) {                              // (fewer are the first CTA's)
    if (some && tid == 0) {
      uint32_t at;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(&s_some)), "r"(0));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(1) : "memory");
    }
    cluster_arrive();
    cluster_wait();
    some = s_some;
  }
  if (cta != 0) return;
  unsigned top = (unsigned)n_free + (unsigned)total;
  if (some) {
    // from the bottom of what is given back upwards: the entries themselves, or what has been written of them
    top = n_free;
    for (unsigned i0 = 0; i0 < (unsigned)total; i0 += PLAN_THREADS) {
      const unsigned i = i0 + tid;
      int page = -1;
      if (i < (unsigned)total) {
        if (room) {
          page = p.free_pages[(unsigned)n_free + i];
        } else {
          const int at = (int)((unsigned)total - 1 - i), b = find_near(ends, p.B, 0, at);
          int32_t* entry = p.page_table + (size_t)b * p.max_pages + pages_of(news[b]) + (at - (b ? ends[b - 1] : 0));
          page = *entry;
          *entry = -1;
        }
      }
      const bool is = can_be_page(page);
      int sum;
      const unsigned to = top + block_scan<PLAN_THREADS>((int)is, red_pages, sum) - 1;
      if (is && to < (unsigned)p.free_cap) p.free_pages[to] = page;
      top += sum;
    }
  }
  if (tid == 0) *p.n_free = (int)min(top, (unsigned)p.free_cap);
}

// ---------------------------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------------------------

struct AppendParams {
  const char *k, *v;
  long long k_row, k_head, v_row, v_head;      // bytes
  const int32_t* slot;
  char *k_pool, *v_pool, *k_min, *k_max;
  int T, H, block;
  long long n_slots;
};

// Smaller / larger of each pair, a NaN if there is one.
__device__ __forceinline__ uint32_t lower(uint32_t a, uint32_t b, bf16) {
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t upper(uint32_t a, uint32_t b, bf16) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t lower(uint32_t a, uint32_t b, float) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
  return __float_as_uint(r);
}
__device__ __forceinline__ uint32_t upper(uint32_t a, uint32_t b, float) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
  return __float_as_uint(r);
}

// A run is what follows one another in the list within one page.  LANES threads own the runs of one head that begin in a window of `block` rows of the
// list, each 16 bytes of the head: a run has one owner, so the page's minimum and maximum need no atomics and do not depend on any
// order.  BATCH rows are in flight at once.  Keys and values are for different threads (blockIdx.y).
// Bound by HBM: 16000 tokens of 8 heads of 128, bf16, 136 MB: 25 us, 5.4 TB/s.  64 tokens 1.8 us.  (More rows in flight, fewer CTAs to an SM: 28 us; copying and summaries by different
// CTAs, the keys read a second time out of L2: 34; windows of fewer rows: 27 to 33.)
template <typename T, int DH>
__global__ void __launch_bounds__(256, 4) kv_append_kernel(const AppendParams p) {
  constexpr int LANES = DH * (int)sizeof(T) / 16, ROW = DH * (int)sizeof(T), BATCH = CERB_PAGE / 4;
  const int lane = threadIdx.x % LANES;
  const long long item = ((long long)blockIdx.x * 256 + threadIdx.x) / LANES;
  const int h = (int)(item % p.H);
  const long long t0 = item / p.H * p.block;
  const bool values = blockIdx.y != 0;
  const char* src = (values ? p.v + h * p.v_head : p.k + h * p.k_head) + lane * 16;
  const long long row = values ? p.v_row : p.k_row;
  char* pool = (values ? p.v_pool : p.k_pool) + lane * 16;
  const bool sums = !values && p.k_min != nullptr;
  const unsigned group = LANES == 32 ? 0xffffffffu : ((1u << LANES) - 1) << ((threadIdx.x & 31) / LANES * LANES);
  griddep_wait();
  auto page_of = [&](long long t) {
    const int s = t >= 0 && t < p.T ? p.slot[t] : -1;
    return s >= 0 && s < p.n_slots ? s / CERB_PAGE : -1;
  };
  // which rows of the window begin a run
  unsigned starts = 0;
#pragma unroll
  for (int w = 0; w < CERB_PAGE; w += LANES) {
    const long long t = t0 + w + lane;
    const int page = w + lane < p.block ? page_of(t) : -1;
    const unsigned mine = __ballot_sync(group, page >= 0 && page_of(t - 1) != page) >> ((threadIdx.x & 31) / LANES * LANES);
    starts |= (LANES == 32 ? mine : mine & ((1u << LANES) - 1)) << w;
  }
  for (; starts; starts &= starts - 1) {
    const long long t = t0 + __ffs(starts) - 1;
    const int page = p.slot[t] / CERB_PAGE;
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo, old_lo = lo, old_hi = lo;
    bool fresh = false, first = true;
    uint4* at = reinterpret_cast<uint4*>(sums ? p.k_min + ((size_t)page * p.H + h) * ROW + lane * 16 : nullptr);
    uint4* at_hi = reinterpret_cast<uint4*>(sums ? p.k_max + ((size_t)page * p.H + h) * ROW + lane * 16 : nullptr);
    if (sums) { old_lo = *at; old_hi = *at_hi; }
    char* to = pool + ((size_t)page * p.H + h) * CERB_PAGE * ROW;
    auto take = [&](const uint4& x, const uint4& y) {
      if (first) { lo = x; hi = y; first = false; return; }
      lo = make_uint4(lower(lo.x, x.x, T()), lower(lo.y, x.y, T()), lower(lo.z, x.z, T()), lower(lo.w, x.w, T()));
      hi = make_uint4(upper(hi.x, y.x, T()), upper(hi.y, y.y, T()), upper(hi.z, y.z, T()), upper(hi.w, y.w, T()));
    };
    for (long long u = t;; u += BATCH) {
      int off[BATCH];
      uint4 x[BATCH];
      int n = 0;
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int s = u + i < p.T ? p.slot[u + i] : -1;
        off[i] = s >= 0 && s / CERB_PAGE == page ? s % CERB_PAGE : -1;
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        if (n == i && off[i] >= 0) ++n;
        if (i < n) x[i] = *reinterpret_cast<const uint4*>(src + (u + i) * row);
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        if (i >= n) continue;
        *reinterpret_cast<uint4*>(to + off[i] * ROW) = x[i];
        if (!sums) continue;
        fresh |= off[i] == 0;
        take(x[i], x[i]);
      }
      if (n < BATCH) break;
    }
    if (!sums) continue;
    if (!fresh) take(old_lo, old_hi);
    *at = lo;
    *at_hi = hi;
  }
}

int check_pages(const cerb_pages* s) {
  if (!s || s->B < 0 || s->max_pages < 1 || s->free_cap < 0) return CERB_E_ARG;
  if ((s->B && (!s->len || !s->page_table)) || (s->free_cap && !s->free_pages) || !s->n_free) return CERB_E_ARG;
  if (s->B > kMaxRequests || s->max_pages > (1 << 26) || (long long)s->B * s->max_pages > 0x7fffffffll) return CERB_E_SHAPE;
  return CERB_OK;
}

PagesParams pages_params(const cerb_pages* s) {
  PagesParams p;
  memset(&p, 0, sizeof(p));
  p.len = s->len;
  p.page_table = s->page_table;
  p.free_pages = s->free_pages;
  p.n_free = s->n_free;
  p.B = s->B;
  p.max_pages = s->max_pages;
  p.free_cap = s->free_cap;
  return p;
}

}  // namespace

}  // namespace cerb

using namespace cerb;

extern "C" {

int cerb_pages_plan(const cerb_pages* s, const int32_t* n_new, int32_t rows, int32_t* slot, int32_t* pos, int32_t* seq, int32_t* row_off,
                    int32_t* granted, void* stream) {
  CERB_TRY(check_pages(s));
  if ((s->B && (!n_new || !granted)) || !row_off || rows < 0 || (rows && (!slot || !pos || !seq))) return CERB_E_ARG;
  if (rows > (1 << 30)) return CERB_E_SHAPE;
  PagesParams p = pages_params(s);
  p.n_new = n_new;
  p.slot = slot;
  p.pos = pos;
  p.seq = seq;
  p.row_off = row_off;
  p.granted = granted;
  p.rows = rows;
  const size_t smem = 4 * (size_t)p.B * sizeof(int);
  cudaStream_t st = (cudaStream_t)stream;
  static std::atomic<uint64_t> done[2];
  if (p.B <= PLAN_FEW && rows <= 2 * PLAN_FEW)
    return launch_pdl(pages_plan_kernel<PLAN_FEW, true>, dim3(1), dim3(PLAN_FEW), smem, st, p) == cudaSuccess ? CERB_OK : CERB_E_CUDA;
  if (rows <= kPlanRowsAlone) {
    CERB_TRY(allow_smem(pages_plan_kernel<PLAN_THREADS, true>, done[0], 4 * kMaxRequests * (int)sizeof(int)));
    return launch_pdl(pages_plan_kernel<PLAN_THREADS, true>, dim3(1), dim3(PLAN_THREADS), smem, st, p) == cudaSuccess ? CERB_OK : CERB_E_CUDA;
  }
  CERB_TRY(allow_smem(pages_plan_kernel<PLAN_THREADS, false>, done[1], 4 * kMaxRequests * (int)sizeof(int)));
  const int ctas = std::min(148, (rows + PLAN_THREADS - 1) / PLAN_THREADS);
  if (launch_pdl(pages_plan_kernel<PLAN_THREADS, false>, dim3((unsigned)ctas), dim3(PLAN_THREADS), smem, st, p) != cudaSuccess) return CERB_E_CUDA;
  return launch_pdl(pages_grant_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, p) == cudaSuccess ? CERB_OK : CERB_E_CUDA;
}

int cerb_pages_trim(const cerb_pages* s, const int32_t* keep, void* stream) {
  CERB_TRY(check_pages(s));
  if (s->B == 0) return CERB_OK;
  if (!keep) return CERB_E_ARG;
  PagesParams p = pages_params(s);
  p.n_new = keep;
  static std::atomic<uint64_t> done[2];
  CERB_TRY(allow_smem(pages_trim_kernel, done[0], 2 * kMaxRequests * (int)sizeof(int)));
  const unsigned ctas = p.B > PLAN_THREADS ? TRIM_WIDE : TRIM_CLUSTER;
  if (ctas > 8) CERB_TRY(allow_wide_clusters(pages_trim_kernel, done[1]));
  return launch_pdl_cluster(pages_trim_kernel, dim3(ctas), dim3(PLAN_THREADS), 2 * (size_t)p.B * sizeof(int), (cudaStream_t)stream, ctas, p) == cudaSuccess
             ? CERB_OK : CERB_E_CUDA;
}

int cerb_kv_append(const cerb_kv_append_args* a, void* stream) {
  if (!a || !a->k_min != !a->k_max) return CERB_E_ARG;
  if (a->T > 0 && (!a->k || !a->v || !a->slot || !a->k_pool || !a->v_pool)) return CERB_E_ARG;
  if ((a->dtype != CERB_F32 && a->dtype != CERB_BF16) || a->T < 0) return CERB_E_ARG;
  if (a->n_kv_heads < 1 || (a->head_dim != 64 && a->head_dim != 128) || a->n_pool_pages < 1 || a->n_pool_pages > (1 << 27) - 1) return CERB_E_SHAPE;
  const int es = a->dtype == CERB_BF16 ? 2 : 4;
  const long long strides[4] = {a->k_row_stride, a->k_head_stride, a->v_row_stride, a->v_head_stride};
  for (long long x : strides)
    if (x * es % 16) return CERB_E_ARG;
  if (((uintptr_t)a->k | (uintptr_t)a->v | (uintptr_t)a->k_pool | (uintptr_t)a->v_pool | (uintptr_t)a->k_min | (uintptr_t)a->k_max) & 15) return CERB_E_ARG;
  if (a->T == 0) return CERB_OK;
  AppendParams p;
  p.k = (const char*)a->k;
  p.v = (const char*)a->v;
  p.k_row = a->k_row_stride * es;
  p.k_head = a->k_head_stride * es;
  p.v_row = a->v_row_stride * es;
  p.v_head = a->v_head_stride * es;
  p.slot = a->slot;
  p.k_pool = (char*)a->k_pool;
  p.v_pool = (char*)a->v_pool;
  p.k_min = (char*)a->k_min;
  p.k_max = (char*)a->k_max;
  p.T = a->T;
  p.H = a->n_kv_heads;
  p.n_slots = (long long)a->n_pool_pages * CERB_PAGE;
  // a token to a group of threads while they all fit the GPU at once, else as many as make it fit, a page at most
  const long long lanes = a->head_dim * es / 16, threads = 2 * (long long)p.T * p.H * lanes, room = 148ll * 512;
  p.block = (int)((threads + room - 1) / room);
  if (p.block > CERB_PAGE) p.block = CERB_PAGE;
  const long long groups = ((long long)p.T + p.block - 1) / p.block * p.H, ctas = (groups * lanes + 255) / 256;
  if (ctas > 0x7fffffffll) return CERB_E_SHAPE;
  const dim3 grid((unsigned)ctas, 2);
  auto kern = a->dtype == CERB_BF16 ? (a->head_dim == 128 ? kv_append_kernel<bf16, 128> : kv_append_kernel<bf16, 64>)
                                    : (a->head_dim == 128 ? kv_append_kernel<float, 128> : kv_append_kernel<float, 64>);
  return launch_pdl(kern, grid, dim3(256), 0, (cudaStream_t)stream, p) == cudaSuccess ? CERB_OK : CERB_E_CUDA;
}

}  // extern "C"
