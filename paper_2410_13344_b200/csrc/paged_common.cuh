// Shared by the kernels that read a paged cache for one new token.  Device code only.
#pragma once

#include "cerb_internal.cuh"

namespace cerb {

// 16 bytes that are read once.  (Not through the read-only path: kernels in front may have written them.)
__device__ __forceinline__ uint4 ld16(const void* src) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(src) : "memory");
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

}  // namespace cerb
