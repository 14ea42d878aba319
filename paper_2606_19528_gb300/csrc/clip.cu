// Global norm of many gradient tensors, and their clipping to a bound:
//   norm = sqrt(sum g^2),  coef = norm > max_norm ? max_norm / norm : 1,  dst = coef * src
// Two launches: the CTAs' sums of squares, then the scaling, each of whose CTAs adds the partial sums up again in
// the same order.  Both are bound by memory.  The tensors' table is a kernel argument: no copy precedes the launches.
#include "common.cuh"
#include "kernels.h"

namespace lora {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = kClipChunk / kThreads;  // elements of a chunk per thread

__device__ __forceinline__ int find_tensor(const ClipBatch& b, int chunk) {
  int lo = 0, hi = b.n;
  while (hi - lo > 1) {
    const int m = (lo + hi) / 2;
    if (b.t[m].chunk_begin <= chunk)
      lo = m;
    else
      hi = m;
  }
  return lo;
}

// Sum over the block's threads; every thread gets it.
__device__ double block_sum(double v) {
  __shared__ double part[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) s += part[w];
  return s;
}

__device__ __forceinline__ float load(const ClipTensor& t, long long i) {
  return t.half ? __bfloat162float(static_cast<const __nv_bfloat16*>(t.src)[i]) : static_cast<const float*>(t.src)[i];
}

__global__ void __launch_bounds__(kThreads) clip_sum_kernel(const __grid_constant__ ClipBatch b,
                                                            double* __restrict__ partial) {
  griddep_wait();
  griddep_launch_dependents();
  double sum = 0.0;
  for (int c = blockIdx.x; c < b.chunks; c += gridDim.x) {
    const ClipTensor& t = b.t[find_tensor(b, c)];
    const long long i0 = (long long)(c - t.chunk_begin) * kClipChunk;
    const int n = (int)min((long long)kClipChunk, t.n - i0);
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const double v = (double)load(t, i0 + i);
      sum += v * v;
    }
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(kThreads) clip_scale_kernel(const __grid_constant__ ClipBatch b,
                                                              const double* __restrict__ partial, int n_partial,
                                                              float max_norm, float* __restrict__ norm_out,
                                                              float* __restrict__ coef_out) {
  griddep_wait();
  griddep_launch_dependents();
  double sum = 0.0;
  for (int i = threadIdx.x; i < n_partial; i += kThreads) sum += partial[i];
  const double norm = sqrt(block_sum(sum));
  // a norm that is not finite (an infinity or a NaN in a gradient) leaves the tensors as they are
  const double exact = isfinite(norm) && norm > (double)max_norm ? (double)max_norm / norm : 1.0;
  const float coef = (float)exact;
  // a coefficient that fp32 would round as a subnormal is applied in two factors
  const float pre = exact < 0x1p-100 ? 0x1p-64f : 1.f, mul = (float)(exact / (double)pre);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *norm_out = (float)norm;
    if (coef_out) *coef_out = coef;
  }
  for (int c = blockIdx.x; c < b.chunks; c += gridDim.x) {
    const ClipTensor& t = b.t[find_tensor(b, c)];
    if (!t.dst || (coef == 1.f && t.dst == t.src)) continue;
    const long long i0 = (long long)(c - t.chunk_begin) * kClipChunk;
    const int n = (int)min((long long)kClipChunk, t.n - i0);
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const float x = load(t, i0 + i), v = x * pre * mul;
      if (t.half)
        static_cast<__nv_bfloat16*>(t.dst)[i0 + i] =
            coef == 1.f ? static_cast<const __nv_bfloat16*>(t.src)[i0 + i] : __float2bfloat16(v);
      else
        static_cast<float*>(t.dst)[i0 + i] = coef == 1.f ? x : v;  // coef 1 keeps a NaN's bits too
    }
  }
}

}  // namespace

int clip_ctas(int chunks, int num_sms) { return chunks < 8 * num_sms ? (chunks > 0 ? chunks : 1) : 8 * num_sms; }

cudaError_t launch_clip_sum(const ClipBatch& b, double* partial, int ctas, cudaStream_t st) {
  return launch_kernel(clip_sum_kernel, dim3(ctas), dim3(kThreads), 0, st, 1, b, partial);
}

cudaError_t launch_clip_scale(const ClipBatch& b, const double* partial, int n_partial, float max_norm, float* norm,
                              float* coef, int ctas, cudaStream_t st) {
  return launch_kernel(clip_scale_kernel, dim3(ctas), dim3(kThreads), 0, st, 1, b, partial, n_partial, max_norm, norm,
                       coef);
}

}  // namespace lora
