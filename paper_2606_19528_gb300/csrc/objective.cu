// Losses over sequences of sampled or preferred tokens, from the tokens' negative log-probabilities:
//   policy_kernel  clipped policy loss with a KL term, one block per sequence
//   pref_kernel    loss of a chosen against a rejected sequence, one block per pair
//   rows_kernel    the loss's sum, the tokens' weights w_t = d loss / d nll_t, and dh_t = w_t * d nll_t / d h_t
// The first launch reads a few bytes per token; the second streams two rows of d bf16 per token and is bound by
// memory.  It needs the first one's sums: a weight depends on its whole sequence or batch.
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "lora.h"

namespace lora {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ T block_sum(T v) {
  __shared__ T part[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  T s = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) s += part[w];
  return s;
}

// Offsets i and i + 1, inside [0, T] and in order whatever the array holds; records ones that are not.
__device__ __forceinline__ void range(const Objective& o, int i, int last, int* lo, int* hi) {
  const int a = o.offsets[i], c = o.offsets[i + 1];
  *lo = min(max(a, 0), o.T);
  *hi = min(max(c, *lo), o.T);
  if (threadIdx.x == 0 && (*lo != a || *hi != c || (i == 0 && a != 0) || (i == last && c != o.T)))
    atomicCAS(o.status, 0, kStatusOffsets);
}

// exp(e) - 1 - e without its cancellation near zero: the series below 1/2 (remainder under 2^-26 of the sum).
__device__ __forceinline__ float exp_minus_line(float e) {
  if (fabsf(e) >= 0.5f) return expm1f(e) - e;
  float s = 1.f;
#pragma unroll
  for (int k = 9; k >= 3; --k) s = fmaf(s, e * (1.f / (float)k), 1.f);
  return 0.5f * e * e * s;
}

__global__ void __launch_bounds__(kThreads) policy_kernel(const __grid_constant__ Objective o) {
  griddep_wait();
  griddep_launch_dependents();
  const int s = blockIdx.x;
  int lo, hi;
  range(o, s, o.groups - 1, &lo, &hi);
  int n = 0;
  for (int t = lo + threadIdx.x; t < hi; t += kThreads) n += !o.mask || o.mask[t] ? 1 : 0;
  n = block_sum(n);
  const double norm = (double)o.scale * (o.reduction == LORA_MEAN_SEQS && n ? 1.0 / ((double)o.groups * n) : 1.0);
  double loss = 0.0, kl_sum = 0.0;
  int clips = 0;
  for (int t = lo + threadIdx.x; t < hi; t += kThreads) {
    float u = 0.f;
    if (!o.mask || o.mask[t]) {
      const float nll = o.nll[t], delta = o.old_nll[t] - nll, A = o.adv[o.per_token ? t : s];
      const bool up = A > 0.f && delta > o.log_high, down = A < 0.f && delta < o.log_low;
      float l;
      if (up || down) {
        l = -A * (up ? 1.f + o.clip_high : 1.f - o.clip_low);
        ++clips;
      } else {
        u = A * expf(delta);
        l = -u;
      }
      loss += (double)l;
      if (o.ref_nll) {
        const float e = nll - o.ref_nll[t], kl = exp_minus_line(e);
        loss += (double)o.beta * kl;
        kl_sum += (double)kl;
        u = fmaf(o.beta, expm1f(e), u);
      }
      u *= (float)norm;
    }
    o.u[t] = u;
  }
  loss = block_sum(loss);
  kl_sum = block_sum(kl_sum);
  clips = block_sum(clips);
  if (threadIdx.x == 0) o.seq[s] = ObjectiveSeq{loss * norm, kl_sum, n, clips};
}

__global__ void __launch_bounds__(kThreads) pref_kernel(const __grid_constant__ Objective o) {
  griddep_wait();
  griddep_launch_dependents();
  const int p = blockIdx.x;
  int lo[2], hi[2];
  range(o, 2 * p, 2 * o.groups - 1, &lo[0], &hi[0]);
  range(o, 2 * p + 1, 2 * o.groups - 1, &lo[1], &hi[1]);
  double R[2];
  double share[2];
  for (int c = 0; c < 2; ++c) {
    double sum = 0.0;
    int n = 0;
    for (int t = lo[c] + threadIdx.x; t < hi[c]; t += kThreads) {
      if (o.mask && !o.mask[t]) continue;
      sum += (o.ref_nll ? (double)o.ref_nll[t] : 0.0) - (double)o.nll[t];
      ++n;
    }
    sum = block_sum(sum);
    n = block_sum(n);
    share[c] = o.mean_tokens && n ? 1.0 / n : 1.0;
    R[c] = sum * share[c];
  }
  const double beta = o.beta, m = beta * (R[0] - R[1]) - (double)o.margin;
  double loss, slope;
  if (o.kind == LORA_PREF_SIGMOID) {
    const double ls = o.smoothing, tail = log1p(exp(-fabs(m)));
    loss = (1.0 - ls) * (tail + fmax(-m, 0.0)) + ls * (tail + fmax(m, 0.0));
    slope = -(1.0 - ls) / (1.0 + exp(m)) + ls / (1.0 + exp(-m));
  } else if (o.kind == LORA_PREF_HINGE) {
    loss = fmax(1.0 - m, 0.0);
    slope = m < 1.0 ? -1.0 : 0.0;
  } else {
    loss = (m - 0.5) * (m - 0.5) / (beta * beta);
    slope = 2.0 * (m - 0.5) / (beta * beta);
  }
  const double norm = (double)o.scale / o.groups;
  for (int c = 0; c < 2; ++c) {
    const float w = (float)((c ? slope : -slope) * beta * norm * share[c]);
    for (int t = lo[c] + threadIdx.x; t < hi[c]; t += kThreads) o.u[t] = o.mask && !o.mask[t] ? 0.f : w;
  }
  if (threadIdx.x == 0) {
    o.seq[p] = ObjectiveSeq{loss * norm, 0.0, 0, 0};
    if (o.rewards) {
      o.rewards[2 * p] = (float)(beta * R[0]);
      o.rewards[2 * p + 1] = (float)(beta * R[1]);
    }
  }
}

__global__ void __launch_bounds__(kThreads) rows_kernel(const __grid_constant__ Objective o) {
  griddep_wait();
  griddep_launch_dependents();
  float inv = 1.f;
  double total = 1.0;
  const bool by_tokens = o.reduction == LORA_MEAN_TOKENS;
  if (by_tokens || blockIdx.x == 0) {
    long long n = 0;
    for (int s = threadIdx.x; s < o.groups; s += kThreads) n += o.seq[s].n;
    total = (double)block_sum(n);
    if (by_tokens && total > 0.0) inv = (float)(1.0 / total);
  }
  if (blockIdx.x == 0) {
    double loss = 0.0, kl = 0.0;
    long long clips = 0;
    for (int s = threadIdx.x; s < o.groups; s += kThreads) {
      loss += o.seq[s].loss;
      kl += o.seq[s].kl;
      clips += o.seq[s].clipped;
    }
    loss = block_sum(loss);
    kl = block_sum(kl);
    clips = block_sum(clips);
    if (threadIdx.x == 0) {
      const double per = total > 0.0 ? 1.0 / total : 0.0;
      *o.loss = (float)(by_tokens ? loss * per : loss);
      if (o.stats) {
        o.stats[0] = (float)(kl * per);
        o.stats[1] = (float)((double)clips * per);
      }
    }
  }
  if (!o.dh && !o.token_weight) return;
  const int lane = threadIdx.x & 31, vecs = o.d / 8;
  for (int t = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); t < o.T; t += gridDim.x * (kThreads / 32)) {
    const float w = o.u[t] * inv;
    if (o.token_weight && lane == 0) o.token_weight[t] = w;
    if (!o.dh) continue;
    const uint4* src = reinterpret_cast<const uint4*>(o.dh_nll + (long long)t * o.d);
    uint4* dst = reinterpret_cast<uint4*>(o.dh + (long long)t * o.d);
    for (int v = lane; v < vecs; v += 32) {
      uint4 r = make_uint4(0u, 0u, 0u, 0u);
      if (w != 0.f) {  // also a NaN; a row of weight zero is zero whatever the row holds
        const uint4 q = src[v];
        const uint32_t in[4] = {q.x, q.y, q.z, q.w};
        uint32_t out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          out[e] = pack_bf16x2(w * __uint_as_float(in[e] << 16), w * __uint_as_float(in[e] & 0xffff0000u));
        r = make_uint4(out[0], out[1], out[2], out[3]);
      }
      dst[v] = r;
    }
  }
}

cudaError_t launch_rows(const Objective& o, int num_sms, cudaStream_t st) {
  const int ctas = o.dh || o.token_weight ? std::min((o.T + 7) / 8, 8 * num_sms) : 1;
  return launch_kernel(rows_kernel, dim3(ctas), dim3(kThreads), 0, st, 1, o);
}

}  // namespace

cudaError_t launch_policy(const Objective& o, int num_sms, cudaStream_t st) {
  const cudaError_t e = launch_kernel(policy_kernel, dim3(o.groups), dim3(kThreads), 0, st, 1, o);
  return e != cudaSuccess ? e : launch_rows(o, num_sms, st);
}

cudaError_t launch_pref(const Objective& o, int num_sms, cudaStream_t st) {
  const cudaError_t e = launch_kernel(pref_kernel, dim3(o.groups), dim3(kThreads), 0, st, 1, o);
  return e != cudaSuccess ? e : launch_rows(o, num_sms, st);
}

}  // namespace lora
