// Sums held as an unevaluated pair of fp32: about 48 bits at fp32's speed.  (FP64 runs at about 2 operations a clock
// and SM on this GPU.)
#pragma once

#include <cuda_runtime.h>

namespace lora {

// hi + lo, |lo| small against |hi|; Pair{} is zero.
struct Pair {
  float hi, lo;

  // x and its addition's rounding error (two-sum)
  __device__ __forceinline__ void add(float x) {
    const float s = hi + x, b = s - hi;
    lo += (hi - (s - b)) + (x - b);
    hi = s;
  }
  __device__ __forceinline__ void add(const Pair& p) {
    add(p.hi);
    lo += p.lo;
  }
  __device__ __forceinline__ Pair times(float x) const {
    Pair r;
    r.hi = hi * x;
    r.lo = isfinite(r.hi) ? fmaf(hi, x, -r.hi) + lo * x : 0.f;
    return r;
  }
  __device__ __forceinline__ Pair over(float x) const {
    Pair r;
    r.hi = hi / x;
    r.lo = isfinite(r.hi) ? (fmaf(-r.hi, x, hi) + lo) / x : 0.f;
    return r;
  }
  // an infinite or undefined sum has no error term
  __device__ __forceinline__ float value() const { return isfinite(hi) ? hi + lo : hi; }
  __device__ __forceinline__ double wide() const { return isfinite(hi) ? (double)hi + (double)lo : (double)hi; }
};

__device__ __forceinline__ Pair warp_sum(Pair p) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Pair q;
    q.hi = __shfl_xor_sync(0xffffffffu, p.hi, o);
    q.lo = __shfl_xor_sync(0xffffffffu, p.lo, o);
    p.add(q);
  }
  return p;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace lora
