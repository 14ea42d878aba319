// Losses over sequences of sampled or preferred tokens, from the tokens' negative log-probabilities:
//   policy_kernel  clipped policy loss with a KL term, one cluster of 1 or 8 CTAs per sequence
//   pref_kernel    loss of a chosen against a rejected sequence, one cluster per pair
//   rows_kernel    the loss's sum, the tokens' weights w_t = d loss / d nll_t, and dh_t = w_t * d nll_t / d h_t
//   few_kernel     all of either loss for few tokens: 3.2 to 3.8 us for 61 of 256
// The first launch reads a few bytes per token and is a chain of latencies (about 4.5 us with the launches); the
// second streams two rows of d bf16 per trainable token, one per masked token, and is bound by memory: 58 us for the
// 352 MB of 49152 tokens of 2048, a quarter of them masked, 0.9 of the copy rate.  It needs the first one's sums (a
// weight depends on its whole sequence or batch), but starts beside it: its first rows are on their way when the sums
// arrive.
//
// Sums over tokens are held as pairs of fp32 (48 bits).
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "lora.h"
#include "pair.cuh"

namespace lora {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBatch = 4;  // tokens of a thread whose loads are in flight together

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}

// Two sums and two counts over the cluster's threads.
struct Totals {
  Pair a, b;
  int n, m;
};

__device__ __forceinline__ Totals warp_totals(Totals v) {
  v.a = warp_sum(v.a);
  v.b = warp_sum(v.b);
  v.n = __reduce_add_sync(0xffffffffu, v.n);
  v.m = __reduce_add_sync(0xffffffffu, v.m);
  return v;
}

// Every thread of the cluster gets the sums over it, added in the order of the warps: each warp's go into its slot of
// every CTA's shared memory (after cluster_begun_arrive() where there are several).
__device__ __forceinline__ Totals cluster_totals(Totals v, Totals* slots) {
  const uint32_t ctas = cluster_size(), rank = ctas > 1 ? cluster_ctarank() : 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  v = warp_totals(v);
  if (ctas > 1) cluster_begun_wait();
  if (lane < (int)ctas) {
    const uint32_t words[6] = {__float_as_uint(v.a.hi), __float_as_uint(v.a.lo), __float_as_uint(v.b.hi),
                               __float_as_uint(v.b.lo), (uint32_t)v.n,           (uint32_t)v.m};
    const uint32_t at = smem_u32(&slots[rank * kWarps + warp]);
    if (ctas > 1) {
      const uint32_t to = mapa_shared(at, lane);
#pragma unroll
      for (int i = 0; i < 6; ++i) st_cluster_u32(to + 4 * i, words[i]);
    } else {
      slots[warp] = v;
    }
  }
  if (ctas > 1)
    cluster_sync_all();
  else
    __syncthreads();
  Totals t{};
  for (int s = lane; s < (int)ctas * kWarps; s += 32) {
    const Totals& q = slots[s];
    t.a.add(q.a);
    t.b.add(q.b);
    t.n += q.n;
    t.m += q.m;
  }
  return warp_totals(t);
}

// Offsets i and i + 1, inside [0, T] and in order whatever the array holds; records ones that are not.
__device__ __forceinline__ void range(const Objective& o, int i, int last, bool records, int* lo, int* hi) {
  const int a = o.offsets[i], c = o.offsets[i + 1];
  *lo = min(max(a, 0), o.T);
  *hi = min(max(c, *lo), o.T);
  if (records && (*lo != a || *hi != c || (i == 0 && a != 0) || (i == last && c != o.T)))
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

// The thread's tokens t0, t0 + stride, .. below hi: their terms added to v (a: losses, b: divergences, n: trainable, m:
// clipped), and the weights u that they have before the norm.
__device__ __forceinline__ void policy_tokens(const Objective& o, int t0, int stride, int hi, float adv_seq, Totals& v,
                                              float (&u)[kBatch]) {
  float nll[kBatch], old[kBatch], ref[kBatch], adv[kBatch];
  bool on[kBatch];
#pragma unroll
  for (int k = 0; k < kBatch; ++k) {
    const int t = t0 + k * stride;
    const int at = min(t, hi - 1);  // a masked token's values are loaded with its mask, and dropped
    on[k] = t < hi && (!o.mask || o.mask[at]);
    nll[k] = o.nll[at];
    old[k] = o.old_nll[at];
    ref[k] = o.ref_nll ? o.ref_nll[at] : 0.f;
    adv[k] = o.per_token ? o.adv[at] : adv_seq;
  }
#pragma unroll
  for (int k = 0; k < kBatch; ++k) {
    u[k] = 0.f;
    if (!on[k]) continue;
    const float delta = old[k] - nll[k], A = adv[k];
    const bool up = A > 0.f && delta > o.log_high, down = A < 0.f && delta < o.log_low;
    float l;
    if (up || down) {
      l = -A * (up ? 1.f + o.clip_high : 1.f - o.clip_low);
      ++v.m;
    } else {
      u[k] = A == 0.f && isfinite(delta) ? 0.f : A * expf(delta);  // also where the exponential is beyond fp32
      l = -u[k];
    }
    if (o.ref_nll) {
      const float e = nll[k] - ref[k], kl = exp_minus_line(e);
      v.b.add(kl);
      if (o.beta != 0.f) u[k] = fmaf(o.beta, expm1f(e), u[k]);
    }
    v.a.add(l);
    ++v.n;
    u[k] *= o.scale;
  }
}

__global__ void __launch_bounds__(kThreads) policy_kernel(const __grid_constant__ Objective o) {
  __shared__ Totals slots[kMaxCluster * kWarps];
  const int ctas = (int)cluster_size(), s = (int)blockIdx.x / ctas;
  if (ctas > 1) cluster_begun_arrive();
  griddep_wait();
  griddep_launch_dependents();
  int lo, hi;
  range(o, s, o.groups - 1, threadIdx.x == 0, &lo, &hi);
  const bool by_seq = o.reduction == LORA_MEAN_SEQS;
  const int stride = ctas * kThreads, first = lo + ((int)blockIdx.x % ctas) * kThreads + (int)threadIdx.x;
  const bool one_batch = hi - lo <= kBatch * stride;
  const float adv_seq = o.per_token ? 0.f : o.adv[s];
  Totals v{};
  float u[kBatch];
  for (int t0 = first; t0 < hi; t0 += kBatch * stride) {
    policy_tokens(o, t0, stride, hi, adv_seq, v, u);
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (t0 + k * stride < hi && (!by_seq || !one_batch)) o.u[t0 + k * stride] = u[k];
  }
  const Totals all = cluster_totals(v, slots);
  if (by_seq && all.n) {
    const float norm = 1.f / ((float)o.groups * (float)all.n);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) u[k] *= norm;  // of the only batch
    if (one_batch) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (first + k * stride < hi) o.u[first + k * stride] = u[k];
    } else {
      for (int t = first; t < hi; t += stride) o.u[t] *= norm;
    }
  } else if (by_seq) {  // no trainable token
    for (int t = first; t < hi; t += stride) o.u[t] = 0.f;
  }
  if (blockIdx.x % ctas == 0 && threadIdx.x == 0) {
    o.n[s] = all.n;
    o.seq[s] = ObjectiveSeq{all.a.hi, all.a.lo, all.b.hi, all.b.lo, all.m};
  }
}

// e^-|m| of a pair: what lo adds is a factor near 1.
__device__ __forceinline__ float exp_neg_abs(const Pair& m) {
  const float hi = fabsf(m.hi);
  return hi > 200.f ? 0.f : expf(-hi) * (1.f + (m.hi < 0.f ? m.lo : -m.lo));
}

// The tokens of a pair: position i counts the first sequence's, then the second's.
struct PairTokens {
  int lo[2], hi[2], n0, total;
  __device__ __forceinline__ void load(const Objective& o, int p, bool records) {
    range(o, 2 * p, 2 * o.groups - 1, records, &lo[0], &hi[0]);
    range(o, 2 * p + 1, 2 * o.groups - 1, records, &lo[1], &hi[1]);
    n0 = hi[0] - lo[0];
    total = n0 + hi[1] - lo[1];
  }
  __device__ __forceinline__ int at(int i) const { return i < n0 ? lo[0] + i : lo[1] + i - n0; }

  // The sums over the thread's positions i0, i0 + stride, .. (a, n: the first sequence's; b, m: the second's).
  __device__ __forceinline__ Totals sums(const Objective& o, int first, int stride) const {
    Totals v{};
    for (int i0 = first; i0 < total; i0 += kBatch * stride) {
      float nll[kBatch], ref[kBatch];
      bool on[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int i = i0 + k * stride, t = at(min(i, total - 1));
        on[k] = i < total && (!o.mask || o.mask[t]);
        nll[k] = o.nll[t];
        ref[k] = o.ref_nll ? o.ref_nll[t] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (!on[k]) continue;
        Pair& sum = i0 + k * stride < n0 ? v.a : v.b;
        sum.add(ref[k]);
        sum.add(-nll[k]);
        ++(i0 + k * stride < n0 ? v.n : v.m);
      }
    }
    return v;
  }
};

// A pair's weights w of either sequence's tokens from its sums; its loss and rewards are written where asked.
__device__ __forceinline__ void pref_pair(const Objective& o, int p, const Totals& all, bool writes, float (&w)[2]) {
  const Pair r0 = (o.mean_tokens && all.n ? all.a.over((float)all.n) : all.a).times(o.beta);
  const Pair r1 = (o.mean_tokens && all.m ? all.b.over((float)all.m) : all.b).times(o.beta);
  Pair m = r0;
  m.add(-r1.hi);
  m.lo -= r1.lo;
  m.add(-o.margin);
  const float mv = m.value();
  m.lo = isfinite(mv) ? (m.hi - mv) + m.lo : 0.f;  // lo below hi's last place again
  m.hi = mv;
  Pair loss{};
  float slope;  // times beta
  if (o.kind == LORA_PREF_SIGMOID) {
    // with e = exp(-|m|): log(1 + exp(-|m|)), and the smaller and the larger of sigmoid(+-m)
    const float e = exp_neg_abs(m), small = e / (1.f + e), large = 1.f / (1.f + e);
    const float ls = o.smoothing, by = mv < 0.f ? ls - 1.f : ls;
    if (by != 0.f) loss = m.times(by);
    loss.add(log1pf(e));
    slope = o.beta * (mv < 0.f ? fmaf(ls, small, (ls - 1.f) * large) : fmaf(ls, large, (ls - 1.f) * small));
  } else if (o.kind == LORA_PREF_HINGE) {
    const float past = (mv - 1.f) + m.lo;  // m - 1; the sign also where m rounds to 1
    if (!(past >= 0.f)) {  // also undefined
      loss = m.times(-1.f);
      loss.add(1.f);
    }
    slope = past < 0.f ? -o.beta : (past >= 0.f ? 0.f : mv);
  } else {
    Pair x = m;
    x.add(-0.5f);
    const float xb = x.value() / o.beta;
    loss = x.over(o.beta).times(xb);
    slope = 2.f * xb;
  }
  const float norm = o.scale / (float)o.groups, by = slope * norm;
  w[0] = o.mean_tokens && all.n ? -by / (float)all.n : -by;
  w[1] = o.mean_tokens && all.m ? by / (float)all.m : by;
  if (!writes) return;
  o.seq[p] = ObjectiveSeq{loss.hi, loss.lo, 0.f, 0.f, 0};
  o.n[p] = all.n + all.m;
  if (o.rewards) {
    o.rewards[2 * p] = r0.value();
    o.rewards[2 * p + 1] = r1.value();
  }
}

__global__ void __launch_bounds__(kThreads) pref_kernel(const __grid_constant__ Objective o) {
  __shared__ Totals slots[kMaxCluster * kWarps];
  __shared__ float s_w[2];
  const int ctas = (int)cluster_size(), p = (int)blockIdx.x / ctas, rank = (int)blockIdx.x % ctas;
  if (ctas > 1) cluster_begun_arrive();
  griddep_wait();
  griddep_launch_dependents();
  PairTokens tokens;
  tokens.load(o, p, threadIdx.x == 0);
  const int stride = ctas * kThreads, first = rank * kThreads + (int)threadIdx.x;
  const Totals all = cluster_totals(tokens.sums(o, first, stride), slots);
  if (threadIdx.x == 0) {
    float w[2];
    pref_pair(o, p, all, rank == 0, w);
    s_w[0] = w[0];
    s_w[1] = w[1];
  }
  __syncthreads();
  for (int i = first; i < tokens.total; i += stride) {
    const int t = tokens.at(i);
    o.u[t] = o.mask && !o.mask[t] ? 0.f : s_w[i < tokens.n0 ? 0 : 1];
  }
}

// The loss and the statistics, by one block, in a fixed order.
__device__ void finish(const Objective& o) {
  __shared__ Pair part[2][kWarps];
  __shared__ long long counts[2][kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, used = min(kWarps, (o.groups + 31) / 32);
  const bool by_seq = o.reduction == LORA_MEAN_SEQS;
  if (warp < used) {
    Pair loss{}, kl{};
    long long n = 0, c = 0;
    for (int s = threadIdx.x; s < o.groups; s += 32 * used) {
      const ObjectiveSeq q = o.seq[s];
      const int tokens = o.n[s];
      Pair l, k;
      l.hi = q.loss_hi, l.lo = q.loss_lo, k.hi = q.kl_hi, k.lo = q.kl_lo;
      if (o.policy && o.ref_nll && o.beta != 0.f) l.add(k.times(o.beta));
      loss.add(by_seq && tokens ? l.over((float)tokens) : l);
      kl.add(k);
      n += tokens;
      c += q.clipped;
    }
    loss = warp_sum(loss);
    kl = warp_sum(kl);
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) {
      n += __shfl_xor_sync(0xffffffffu, n, i);
      c += __shfl_xor_sync(0xffffffffu, c, i);
    }
    if (lane == 0) {
      part[0][warp] = loss;
      part[1][warp] = kl;
      counts[0][warp] = n;
      counts[1][warp] = c;
    }
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  Pair loss = part[0][0], kl = part[1][0];
  long long n = counts[0][0], c = counts[1][0];
  for (int w = 1; w < used; ++w) {
    loss.add(part[0][w]);
    kl.add(part[1][w]);
    n += counts[0][w];
    c += counts[1][w];
  }
  const float tokens = (float)max(n, 1ll);
  if (o.reduction == LORA_MEAN_TOKENS) loss = loss.over(tokens);
  if (by_seq || !o.policy) loss = loss.over((float)o.groups);
  *o.loss = loss.value() * o.scale;
  if (o.stats) {
    o.stats[0] = kl.over(tokens).value();
    o.stats[1] = (float)c / tokens;
  }
}

// Trainable tokens of the batch; every thread gets it.
__device__ __forceinline__ long long count_tokens(const Objective& o) {
  __shared__ long long part[kWarps];
  long long n = 0;
  for (int s = threadIdx.x; s < o.groups; s += kThreads) n += o.n[s];
#pragma unroll
  for (int i = 16; i > 0; i >>= 1) n += __shfl_xor_sync(0xffffffffu, n, i);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) n += part[w];
  return n;
}

constexpr int kVecs = 4;               // 16-byte vectors of a lane
constexpr int kPartVecs = 32 * kVecs;  // of a part

// A lane's vectors of a part times w, the token's weight; a row of weight zero is zero whatever it holds.
__device__ __forceinline__ void store_part(const Objective& o, int t, int part, int vecs, float w,
                                           const uint4 (&q)[kVecs]) {
  uint4* dst = reinterpret_cast<uint4*>(o.dh + (long long)t * o.d);
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const int v = (part * kVecs + k) * 32 + (int)(threadIdx.x & 31);
    if (v >= vecs) continue;
    uint4 out = make_uint4(0u, 0u, 0u, 0u);
    if (w != 0.f) {
      const uint32_t in[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
      uint32_t x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[e] = pack_bf16x2(w * __uint_as_float(in[e] << 16), w * __uint_as_float(in[e] & 0xffff0000u));
      out = make_uint4(x[0], x[1], x[2], x[3]);
    }
    __stcs(dst + v, out);
  }
}

// Block 0 finishes the loss.  The others' warps take parts of rows, each through a ring of bulk copies of its own:
// the copies need no registers, so that 192 KB per SM are on their way while the first launch still runs.  16384
// tokens of 3072 for 32 pairs take 29.1 us as four blocks of 8 warps by 3 slots per SM, 30.1 as two by 6, 28.7 as six
// by 2; 49152 tokens of 2048 take 63.1, 63.7 and 64.6; 4096 of 3072 take 8.6, 9.4 and 9.0.  Loads one part ahead
// into registers, four blocks per SM: 31.3, 63 and 9.4.
constexpr int kSlots = 3;              // parts of a warp
constexpr int kRowCtas = 4;            // per SM
constexpr uint32_t kPartBytes = 16u * kPartVecs;
constexpr uint32_t kRowsSmem = kWarps * kSlots * (kPartBytes + 8u);
constexpr long long kDrainNs = 200000000;

__global__ void __launch_bounds__(kThreads, kRowCtas) rows_kernel(const __grid_constant__ Objective o) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ volatile int s_abort;
  if (blockIdx.x == 0) {
    griddep_wait();
    griddep_launch_dependents();
    finish(o);
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const WaitCtl wait{o.status, o.limit_ns};
  const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * kSlots) * kPartBytes;
  const uint32_t bars = smem_u32(smem) + (uint32_t)(kWarps * kSlots) * kPartBytes + (uint32_t)(warp * kSlots) * 8u;
  if (o.dh && lane < kSlots) mbar_init(bars + 8 * lane, 1);
  if (threadIdx.x == 0) s_abort = 0;
  fence_mbar_init();
  __syncthreads();

  const int vecs = o.dh ? o.d / 8 : 0, parts = o.dh ? (vecs + kPartVecs - 1) / kPartVecs : 1;
  const long long warps = ((long long)gridDim.x - 1) * kWarps, w0 = ((long long)blockIdx.x - 1) * kWarps + warp;
  // The warp's i-th part; lane l holds those with i % 32 == l, of these 32 and the next.
  struct Part {
    int t, part;
    bool copied;
    float u;
  };
  auto place = [&](long long i) {
    const long long id = w0 + i * warps, t = id / parts;
    return Part{t < o.T ? (int)t : o.T, (int)(id - t * parts), false, 0.f};
  };
  auto weigh = [&](Part& p) { p.u = p.t < o.T ? o.u[p.t] : 0.f; };
  auto copy = [&](const Part& p, int slot) {
    const int n = min(kPartVecs, vecs - p.part * kPartVecs);
    mbar_arrive_expect_tx(bars + 8 * slot, 16u * n);
    bulk_load(ring + slot * kPartBytes, o.dh_nll + (long long)p.t * o.d + (long long)p.part * (8 * kPartVecs), 16u * n,
              bars + 8 * slot);
  };
  Part cur = place(lane);
  // the mask and the rows were written before the first launch of the call began
  if (o.dh && lane < kSlots && cur.t < o.T && (!o.mask || o.mask[cur.t])) {
    copy(cur, lane);
    cur.copied = true;
  }
  uint32_t pending = __ballot_sync(0xffffffffu, cur.copied);  // bit s: a copy is on its way to slot s
  uint32_t phases = 0;                                         // bit s: the parity of its wait
  griddep_wait();
  griddep_launch_dependents();
  weigh(cur);
  float inv = 1.f;
  if (o.reduction == LORA_MEAN_TOKENS) {
    const long long n = count_tokens(o);
    inv = n ? 1.f / (float)n : 1.f;
  }
  if (o.dh && lane >= kSlots) cur.copied = cur.u != 0.f;  // also a NaN; a row of weight zero is not read
  int slot = 0;
  bool more = true;
  for (long long base = 0; more; base += 32) {
    Part nxt = place(base + 32 + lane);
    weigh(nxt);
    if (o.dh) nxt.copied = nxt.u != 0.f;
    for (int k = 0; k < 32; ++k) {
      const int t = __shfl_sync(0xffffffffu, cur.t, k), part = __shfl_sync(0xffffffffu, cur.part, k);
      const float w = __shfl_sync(0xffffffffu, cur.u, k) * inv;
      const bool copied = __shfl_sync(0xffffffffu, (int)cur.copied, k);
      more = t < o.T;
      if (!more) break;
      if (o.token_weight && part == 0 && lane == 0) o.token_weight[t] = w;
      if (!o.dh) continue;
      uint4 r[kVecs] = {};
      if (copied) {
        more = __all_sync(0xffffffffu, mbar_wait(bars + 8 * slot, (phases >> slot) & 1u, wait, &s_abort));
        if (!more) break;
        phases ^= 1u << slot;
        pending &= ~(1u << slot);
#pragma unroll
        for (int q = 0; q < kVecs; ++q)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(r[q].x), "=r"(r[q].y), "=r"(r[q].z), "=r"(r[q].w)
                       : "r"(ring + slot * kPartBytes + 16u * (uint32_t)(32 * q + lane))
                       : "memory");
        __syncwarp();
      }
      // the part kSlots on takes the slot
      const bool refill = lane == ((k + kSlots) & 31) && (k + kSlots < 32 ? cur : nxt).copied;
      if (refill) copy(k + kSlots < 32 ? cur : nxt, slot);
      if (__any_sync(0xffffffffu, refill)) pending |= 1u << slot;
      store_part(o, t, part, vecs, w, r);
      if (++slot == kSlots) slot = 0;
    }
    if (more) cur = nxt;
  }
  // not empty only after a wait that gave up: no copy outlives the block's shared memory (bounded)
  for (int s = 0; s < kSlots; ++s)
    if ((pending >> s) & 1u) mbar_wait_drain(bars + 8 * s, (phases >> s) & 1u, kDrainNs);
}

// Few tokens: one launch.  Every block computes all weights, a warp per sequence or pair, and scales its own rows;
// block 0 finishes the loss instead.
constexpr int kFewTokens = 256, kFewGroups = 32, kFewWarps = 16;

__global__ void __launch_bounds__(32 * kFewWarps) few_kernel(const __grid_constant__ Objective o) {
  __shared__ float s_u[kFewTokens];
  __shared__ int s_n[kFewWarps];
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int vecs = o.dh ? o.d / 8 : 0, parts = o.dh ? (vecs + kPartVecs - 1) / kPartVecs : 1;
  const int warps = ((int)gridDim.x - 1) * kFewWarps, w0 = ((int)blockIdx.x - 1) * kFewWarps + warp;
  const bool by_seq = o.reduction == LORA_MEAN_SEQS, writes = blockIdx.x == 0 && lane == 0;
  uint4 q[kVecs];
  auto fetch = [&](int t, int part) {
    const uint4* src = reinterpret_cast<const uint4*>(o.dh_nll + (long long)t * o.d);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int v = (part * kVecs + k) * 32 + lane;
      q[k] = v < vecs ? __ldcs(src + v) : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  // the warp's first part is on its way while the weights are computed
  const int first = w0 / parts;
  const bool ahead = o.dh && blockIdx.x && first < o.T && (!o.mask || o.mask[first]);
  if (ahead) fetch(first, w0 % parts);
  int trainable = 0;
  for (int g = warp; g < o.groups; g += kFewWarps) {
    if (o.policy) {
      int lo, hi;
      range(o, g, o.groups - 1, writes, &lo, &hi);
      const float adv = o.per_token ? 0.f : o.adv[g];
      Totals v{};
      for (int t0 = lo + lane; t0 < hi; t0 += kBatch * 32) {
        float u[kBatch];
        policy_tokens(o, t0, 32, hi, adv, v, u);
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
          if (t0 + 32 * k < hi) s_u[t0 + 32 * k] = u[k];
      }
      v = warp_totals(v);
      if (by_seq && v.n) {
        const float norm = 1.f / ((float)o.groups * (float)v.n);
        for (int t = lo + lane; t < hi; t += 32) s_u[t] *= norm;
      }
      trainable += v.n;
      if (writes) {
        o.n[g] = v.n;
        o.seq[g] = ObjectiveSeq{v.a.hi, v.a.lo, v.b.hi, v.b.lo, v.m};
      }
    } else {
      PairTokens tokens;
      tokens.load(o, g, writes);
      const Totals v = warp_totals(tokens.sums(o, lane, 32));
      float w[2];
      pref_pair(o, g, v, writes, w);
      for (int i = lane; i < tokens.total; i += 32) {
        const int t = tokens.at(i);
        s_u[t] = o.mask && !o.mask[t] ? 0.f : w[i < tokens.n0 ? 0 : 1];
      }
    }
  }
  if (lane == 0) s_n[warp] = trainable;
  __syncthreads();
  if (blockIdx.x == 0) {
    finish(o);
    return;
  }
  float inv = 1.f;
  if (o.reduction == LORA_MEAN_TOKENS) {
    int n = 0;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) n += s_n[w];
    inv = n ? 1.f / (float)n : 1.f;
  }
  for (int i = w0; i < o.T * parts; i += warps) {
    const int t = i / parts, part = i % parts;
    const float u = s_u[t], w = u * inv;
    if (o.token_weight && part == 0 && lane == 0) o.token_weight[t] = w;
    if (!o.dh) continue;
    if (u != 0.f && !(ahead && i == w0)) fetch(t, part);
    store_part(o, t, part, vecs, w, q);
  }
}

// Eight CTAs share a group where groups hold over a token per thread on average (the longest of an uneven batch
// several times that, and the launch ends with it) and all CTAs run at once.
int cluster_for(const Objective& o, int num_sms) {
  return o.T / o.groups > kThreads && o.groups <= num_sms ? kMaxCluster : 1;
}

// Blocks of rows: a warp for each part, up to `most` blocks.
int row_ctas(const Objective& o, int warps, int most) {
  if (!o.dh && !o.token_weight) return 0;
  const long long parts = o.dh ? (o.d / 8 + kPartVecs - 1) / kPartVecs : 1;
  return (int)std::min<long long>((o.T * parts + warps - 1) / warps, most);
}

// One launch or two, the GPU alone and calls in a row (us): 61 tokens of 256 in 4 sequences 3.2 and 4.3, 3.8 and 5.5; 256
// of 1024 in one 5.0 and 4.6, 5.3 and 5.5, in 32 5.1 and 4.8, 5.3 and 5.5, in 64 4.8 and 4.8, 5.4 and 5.5; 512 of 2048
// in 4 4.9 and 4.6, 5.2 and 5.4; 1024 of 2048 in 8 6.0 and 4.9, 6.1 and 5.6, in one 10.3 and 5.2.
bool few_tokens(const Objective& o) { return o.T <= kFewTokens && o.groups <= kFewGroups; }

cudaError_t launch_few(const Objective& o, int num_sms, cudaStream_t st) {
  return launch_kernel(few_kernel, dim3(1 + row_ctas(o, kFewWarps, 2 * num_sms - 1)), dim3(32 * kFewWarps), 0, st, 1, o);
}

cudaError_t launch_rows(const Objective& o, int num_sms, cudaStream_t st) {
  const int ctas = row_ctas(o, kWarps, kRowCtas * num_sms - 1);  // and block 0
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = set_smem_once(rows_kernel, kRowsSmem, done);
  if (e != cudaSuccess) return e;
  return launch_kernel(rows_kernel, dim3(1 + ctas), dim3(kThreads), o.dh ? kRowsSmem : 0, st, 1, o);
}

}  // namespace

cudaError_t launch_policy(const Objective& o, int num_sms, cudaStream_t st) {
  if (few_tokens(o)) return launch_few(o, num_sms, st);
  const int c = cluster_for(o, num_sms);
  const cudaError_t e = launch_kernel(policy_kernel, dim3(o.groups * c), dim3(kThreads), 0, st, c, o);
  return e != cudaSuccess ? e : launch_rows(o, num_sms, st);
}

cudaError_t launch_pref(const Objective& o, int num_sms, cudaStream_t st) {
  if (few_tokens(o)) return launch_few(o, num_sms, st);
  const int c = cluster_for(o, num_sms);
  const cudaError_t e = launch_kernel(pref_kernel, dim3(o.groups * c), dim3(kThreads), 0, st, c, o);
  return e != cudaSuccess ? e : launch_rows(o, num_sms, st);
}

}  // namespace lora
