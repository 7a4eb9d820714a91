// Shared by the kernels that read a paged cache for one new token.
#pragma once

#include "cerb_internal.cuh"

namespace cerb {

constexpr int kMaxList = 1 << 30;       // entries of a list of pages: its indices are ints that step past its end

// 16 bytes that are read once.  (Not through the read-only path: kernels in front may have written them.)
__device__ __forceinline__ uint4 ld16(const void* src) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(src) : "memory");
  return r;
}

// Pairs of fp32.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 pair_of(float x, float y) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ f32x2 twice(float x) { return pair_of(x, x); }
__device__ __forceinline__ float2 parts_of(f32x2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
  return r;
}

// Sums over a warp's lanes of N values each, by halving: every exchange carries half of what is left, as many shuffles as values.  Afterwards lane i has
// in x[0 .. R-1], R = N / 32, the sums of the values i R .., with N < 32 in x[0] that of the value i / (32 / N).
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

// The items of all sequences one after another (items(b) of sequence b), cut into equal shares.
struct Share {
  long long begin, end, size;   // items; of every share
  int b;                        // the sequence that begin lies in,
  long long off;                // and where in it
};
// Share `index` of `shares`, each of min_share items at least, or of what one of the `units` has in the mean where that is less: short units are not put one behind
// another while there are CTAs for them.  By a warp, which sums the items up for itself: a few hundred sequences
// are a few loads to a lane, and no barrier.
template <typename F>
__device__ __forceinline__ Share share_of(int B, F items, int index, int shares, int min_share, long long units) {
  const int lane = threadIdx.x & 31, per = (B + 31) / 32, b0 = min(B, lane * per), b1 = min(B, b0 + per);
  long long mine = 0;
#pragma unroll 4
  for (int b = b0; b < b1; ++b) mine += items(b);
  long long sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += u;
  }
  const long long total = __shfl_sync(0xffffffffu, sum, 31);
  Share s;
  const long long even = total >> 32 ? (total + shares - 1) / shares : (unsigned)total / (unsigned)shares + ((unsigned)total % (unsigned)shares != 0);
  s.size = max(even, total >= min_share * units ? (long long)min_share : (long long)max(1u, (unsigned)total / (unsigned)units));
  s.begin = min(total, s.size * index);
  s.end = min(total, s.begin + s.size);
  const bool here = s.begin >= sum - mine && s.begin < sum;
  long long at = sum - mine;
  int b = b0;
  if (here)
    for (;; ++b) {
      const long long n = items(b);
      if (s.begin < at + n) break;
      at += n;
    }
  const int from = max(__ffs(__ballot_sync(0xffffffffu, here)) - 1, 0);
  s.b = __shfl_sync(0xffffffffu, b, from);
  s.off = s.begin - __shfl_sync(0xffffffffu, at, from);
  return s;
}

}  // namespace cerb
