// Small device helpers shared by the kernels of the library.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace af {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// 2^x by the hardware approximation (about 2^-22 relative; denormal results flush to zero).
__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// For a kernel launched with launch_overlapped (common.cuh): it may start while its predecessor in the stream still
// runs, and touches no memory before this has returned (by then everything earlier is complete and visible).  Every
// thread that reads or writes global memory calls it.  Without that kind of launch it does nothing.
__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Lets such a successor start once every block has called this or ended.
__device__ __forceinline__ void let_successor_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Two floats rounded to nearest-even bf16, packed low | high.
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}

// Sequence of a packed token: the largest j in [0, B) with cu[j] <= t  (cu non-decreasing,
// cu[0] = 0, t < cu[B]).  Bounded by log2 B steps whatever cu holds.
__device__ __forceinline__ int find_seq(const int32_t* __restrict__ cu, int B, int t) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(cu + mid) <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// The same search done by one warp, 32 probes per step (2 steps for B = 512, 4 for B = 10^6).
__device__ __forceinline__ int find_seq_warp(const int32_t* __restrict__ cu, int B, int t, int lane) {
  int lo = 0, hi = B;  // invariant: cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int span = hi - lo;
    const int step = (span + 31) / 32;
    const int probe = lo + (lane + 1) * step;  // probes lo+step, lo+2 step, ...
    const bool le = probe < hi && __ldg(cu + probe) <= t;
    const unsigned m = __ballot_sync(0xffffffffu, le);
    const int k = __popc(m);                   // probes are ordered, so the set bits are a prefix
    const int nlo = lo + k * step;
    const int nhi = nlo + step < hi ? nlo + step : hi;
    lo = nlo; hi = nhi;
  }
  return lo;
}

}  // namespace af
