// Global norm of many gradient tensors, and their clipping to a bound:
//   norm = sqrt(sum g^2),  coef = norm > max_norm ? max_norm / norm : 1,  dst = coef * src
//
// A warp takes a piece of 1024 elements (4 KB of fp32) at a time, in two halves, the next half's loads issued before
// one is used; the pieces are dealt to the CTAs in equal contiguous runs.  Small calls run as one launch, many tensors
// as two:
//   clip_one_kernel    one cluster, a piece per warp: the elements stay in registers between the sum and the scaling,
//                      the CTAs exchange their sums through distributed shared memory
//   clip_sum_kernel    the CTAs' sums of squares, one CTA per SM
//   clip_scale_kernel  every CTA adds these up again in the same order, then scales, from the last piece to the first:
//                      what was read last is still in L2
// Many tensors are bound by memory: a read for the norm, a read from L2 or HBM and a write for the scaling.  What the
// sum reads last stays in L2, all else is asked to leave first (28 layers of 16 tensors, 97 MB: 42.0 us call after
// call, 45.0 where nothing was in L2 before; 194 MB at the copy rate take 28.7, 291 take 43).  Few tensors are bound by
// the chain launch, load, sum, exchange, store: 4.0 us for four tensors, 0.66 MB.
// FP64 is scarce on this GPU (about 2 operations a clock and SM), so a lane's 16 squares are summed in fp32 and these
// sums as pairs of fp32; only the warps' sums are added in fp64.  The tensors' table is a kernel argument: no copy
// precedes the launches.
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "pair.cuh"

namespace lora {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kScaleWarps = 16;  // of the scaling, one CTA per SM: their registers hold what is on its way
constexpr int kOneCtas = 16, kOneWarps = 16;  // of the single cluster, which holds a piece per warp

// A piece's place: the elements before the first 16-byte boundary of src (head), the vectors behind them, the rest.
struct Piece {
  const uint8_t* src;
  uint8_t* dst;  // of the piece's first element; null: not written
  int n, head, vecs;
  bool half, same;  // bf16; dst is src
};

__device__ __forceinline__ Piece piece_of(const ClipTensor& t, int c) {
  Piece p;
  p.half = t.half;
  const int shift = p.half ? 1 : 2;  // of an element's size
  const long long i0 = (long long)(c - t.chunk_begin) * kClipChunk;
  p.n = (int)min((long long)kClipChunk, t.n - i0);
  p.src = static_cast<const uint8_t*>(t.src) + (i0 << shift);
  p.dst = t.dst ? static_cast<uint8_t*>(t.dst) + (i0 << shift) : nullptr;
  p.same = t.dst == t.src;
  p.head = min(p.n, (int)(-reinterpret_cast<uintptr_t>(p.src) & 15) >> shift);
  p.vecs = (p.n - p.head) >> (4 - shift);
  return p;
}

// Last tensor of t[0 .. n) whose pieces begin at or before c.
template <typename Table>
__device__ __forceinline__ int find_tensor(const Table& b, int c) {
  int lo = 0, hi = b.n;
  while (hi - lo > 1) {
    const int m = (lo + hi) / 2;
    if (b.t[m].chunk_begin <= c)
      lo = m;
    else
      hi = m;
  }
  return lo;
}

constexpr int kVecs = kClipChunk / 8 / 32;  // 16-byte vectors of a lane in half a piece (all of it with bf16)

// A lane's part of half a piece: every 32nd vector; with the first half, an element of the head or of the rest.
struct Held {
  uint4 v[kVecs];
  uint32_t edge;  // as fp32
};

// The element of the head or the rest that a lane holds, or -1.
__device__ __forceinline__ int edge_index(const Piece& p, int lane) {
  const int body = p.vecs << (p.half ? 3 : 2), i = lane < p.head ? lane : body + lane;
  return i < p.n ? i : -1;
}

// L2 policies: what stays for the scaling, and what is read for the last time or will not stay anyway.  What stays has the
// normal priority: lines read as evict_last held on to L2 long after the call, and the calls behind it paid for them (a
// training layer of 256 tokens 124.1 for 122.8 us, the second of two copies of 40 MB 17.5 for 14.3), while the call
// itself took the same time.
__device__ __forceinline__ uint64_t policy_keep() {
  uint64_t v;
  asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(v));
  return v;
}
__device__ __forceinline__ uint64_t policy_pass() {
  uint64_t v;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(v));
  return v;
}
__device__ __forceinline__ uint4 load_vec(const uint4* p, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p), "l"(policy)
               : "memory");
  return v;
}

template <int PART>
__device__ __forceinline__ void load_piece(const Piece& p, int lane, Held& h, uint64_t policy) {
  const uint4* v = reinterpret_cast<const uint4*>(p.src + (p.head << (p.half ? 1 : 2))) + lane + 32 * kVecs * PART;
  const int left = p.vecs - lane - 32 * kVecs * PART;
#pragma unroll
  for (int q = 0; q < kVecs; ++q) h.v[q] = 32 * q < left ? load_vec(v + 32 * q, policy) : make_uint4(0u, 0u, 0u, 0u);
  h.edge = 0u;
  if (PART == 0) {
    const int e = edge_index(p, lane);
    if (e >= 0)
      h.edge = p.half ? (uint32_t) reinterpret_cast<const uint16_t*>(p.src)[e] << 16
                      : reinterpret_cast<const uint32_t*>(p.src)[e];
  }
}

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Sum of (scale x)^2 over the lane's elements.
template <bool HALF, bool SCALED>
__device__ __forceinline__ float squares(const Held& h, float scale) {
  auto of = [&](float x, float s) {
    if (SCALED) x *= scale;
    return fmaf(x, x, s);
  };
  float s[4] = {of(__uint_as_float(h.edge), 0.f), 0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < kVecs; ++q) {
    const uint32_t w[4] = {h.v[q].x, h.v[q].y, h.v[q].z, h.v[q].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (HALF) {
        s[e] = of(lo_bf16(w[e]), s[e]);
        s[e] = of(hi_bf16(w[e]), s[e]);
      } else {
        s[e] = of(__uint_as_float(w[e]), s[e]);
      }
    }
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// A lane's sum of squares, where fp32 forms them without loss: each half piece's sum between 2^-60 and 2^100, or of
// zeros alone.  Elsewhere `lost` is set, and slow_squares() takes all of the warp's pieces again.
struct Squares {
  Pair sum{};
  bool lost = false;
  __device__ __forceinline__ void add(const Piece& p, const Held& h) {
    const float s = p.half ? squares<true, false>(h, 1.f) : squares<false, false>(h, 1.f);
    if (s >= 0x1p-60f && s <= 0x1p100f) {
      sum.add(s);
      return;
    }
    uint32_t any = h.edge;
#pragma unroll
    for (int q = 0; q < kVecs; ++q) any |= h.v[q].x | h.v[q].y | h.v[q].z | h.v[q].w;
    lost = lost || s != 0.f || (any & (p.half ? 0x7fff7fffu : 0x7fffffffu)) != 0u;  // but for signs
  }
};

// Half a piece's squares from elements scaled by a power of two: 2^60 twice brings the smallest subnormal's square into
// fp32's range, 2^-80 the largest element's.
__device__ __forceinline__ double scaled_squares(const Held& h, bool half) {
  auto of = [&](float scale) { return half ? squares<true, true>(h, scale) : squares<false, true>(h, scale); };
  float s = of(1.f);
  if (s >= 0x1p-60f && s <= 0x1p100f) return (double)s;
  if (!(s < 0x1p-60f)) return (double)of(0x1p-80f) * 0x1p160;
  s = of(0x1p60f);
  return s >= 0x1p-60f ? (double)s * 0x1p-120 : (double)of(0x1p120f) * 0x1p-240;
}

// A lane's sum over pieces c, c + kWarps, .. below c1, whatever the elements.
template <typename Table>
__device__ __noinline__ double slow_squares(const Table& b, int c, int c1) {
  const int lane = threadIdx.x & 31;
  const uint64_t pass = policy_pass();
  double sum = 0.0;
  for (; c < c1; c += kWarps) {
    const Piece p = piece_of(b.t[find_tensor(b, c)], c);
    Held h;
    load_piece<0>(p, lane, h, pass);
    sum += scaled_squares(h, p.half);
    load_piece<1>(p, lane, h, pass);
    sum += scaled_squares(h, p.half);
  }
  return sum;
}

// The warp's sum over its pieces c, c + kWarps, .. below c1.
template <typename Table>
__device__ __forceinline__ double warp_total(const Squares& s, const Table& b, int c, int c1) {
  return __any_sync(0xffffffffu, s.lost) ? warp_sum(slow_squares(b, c, c1)) : warp_sum(s.sum).wide();
}

struct Coef {
  float coef, pre, mul;
};

// norm = sqrt(total) and the coefficient in fp32, total brought to [1, 4) by a power of four 4^k first.  A norm that is not
// finite (an infinity or a NaN in a gradient) leaves the tensors as they are.  A coefficient that fp32 would round as
// a subnormal is applied in two factors.
__device__ __forceinline__ Coef coef_of(double total, float max_norm, float* norm_out, float* coef_out, bool writes) {
  Coef c{1.f, 1.f, 1.f};
  float norm = (float)total;
  if (isfinite(total) && total > 0.0) {
    const int k = (((__double2hiint(total) >> 20) & 0x7ff) - 1023) >> 1;
    const float root = sqrtf((float)__hiloint2double(__double2hiint(total) - (2 * k << 20), __double2loint(total)));
    norm = ldexpf(root, k);
    // norm > max_norm, also where it is beyond fp32
    if (norm > max_norm || (isinf(norm) && !isinf(max_norm))) {
      const float q = max_norm / root;  // coef = q 2^-k
      c.coef = ldexpf(q, -k);
      c.pre = c.coef < 0x1p-100f ? 0x1p-64f : 1.f;
      c.mul = ldexpf(q, c.coef < 0x1p-100f ? 64 - k : -k);
    }
  }
  if (writes) {
    *norm_out = norm;
    if (coef_out) *coef_out = c.coef;
  }
  return c;
}

__device__ __forceinline__ uint16_t half_bits(float x) { return __bfloat16_as_ushort(__float2bfloat16(x)); }

// Elements [i0, i1) of a piece whose destination lies differently from its source against 16 bytes: one by one, read
// again so that a warp's stores are consecutive (the vectors' elements would touch each sector four or eight times).
template <bool HALF>
__device__ __noinline__ void store_apart(const uint8_t* src, uint8_t* dst, int i0, int i1, float pre, float mul,
                                         bool copy) {
  constexpr int kBatch = 16;
  for (int i = i0 + (int)(threadIdx.x & 31); i < i1; i += 32 * kBatch) {
    uint32_t v[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int at = min(i + 32 * k, i1 - 1);
      v[k] = HALF ? (uint32_t) reinterpret_cast<const uint16_t*>(src)[at] : reinterpret_cast<const uint32_t*>(src)[at];
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int at = i + 32 * k;
      if (at >= i1) break;
      if (HALF)
        reinterpret_cast<uint16_t*>(dst)[at] = copy ? (uint16_t)v[k] : half_bits(__uint_as_float(v[k] << 16) * pre * mul);
      else
        reinterpret_cast<uint32_t*>(dst)[at] = copy ? v[k] : __float_as_uint(__uint_as_float(v[k]) * pre * mul);
    }
  }
}

template <bool HALF, int PART>
__device__ __forceinline__ void store_scaled(const Piece& p, int lane, const Held& h, const Coef& c) {
  const bool copy = c.coef == 1.f;  // also keeps a NaN's bits
  constexpr int kPer = HALF ? 8 : 4, kShift = HALF ? 1 : 2;
  uint8_t* body = p.dst + (p.head << kShift);
  const int first = 32 * kVecs * PART;  // vector of the part
  if ((reinterpret_cast<uintptr_t>(body) & 15) == 0 && c.pre == 1.f) {
    const int left = p.vecs - lane - first;
    uint4* o = reinterpret_cast<uint4*>(body) + lane + first;
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
      uint32_t w[4] = {h.v[q].x, h.v[q].y, h.v[q].z, h.v[q].w};
      if (!copy) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = HALF ? pack_bf16x2(lo_bf16(w[e]) * c.mul, hi_bf16(w[e]) * c.mul)
                      : __float_as_uint(__uint_as_float(w[e]) * c.mul);
      }
      if (32 * q < left) __stcs(o + 32 * q, make_uint4(w[0], w[1], w[2], w[3]));
    }
  } else {
    store_apart<HALF>(p.src, p.dst, p.head + first * kPer, p.head + min(p.vecs, first + 32 * kVecs) * kPer, c.pre, c.mul,
                      copy);
  }
  if (PART != 0) return;
  const int e = edge_index(p, lane);
  if (e < 0) return;
  const float x = __uint_as_float(h.edge);
  if (HALF)
    reinterpret_cast<uint16_t*>(p.dst)[e] = copy ? (uint16_t)(h.edge >> 16) : half_bits(x * c.pre * c.mul);
  else
    reinterpret_cast<float*>(p.dst)[e] = copy ? x : x * c.pre * c.mul;
}

template <int PART>
__device__ __forceinline__ void store_piece(const Piece& p, int lane, const Held& h, const Coef& c) {
  if (!p.dst || (c.coef == 1.f && p.same)) return;
  if (p.half)
    store_scaled<true, PART>(p, lane, h, c);
  else
    store_scaled<false, PART>(p, lane, h, c);
}

// The CTA's sum of the warps', in warp 0; one barrier.
template <int WARPS>
__device__ __forceinline__ double cta_sum(double v, double* part) {
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  return threadIdx.x < 32 ? warp_sum(threadIdx.x < WARPS ? part[threadIdx.x] : 0.0) : 0.0;
}

// The run of pieces [c0, c1) that is this CTA's; its warps take them in turn.
__device__ __forceinline__ void run_of(int chunks, int* c0, int* c1) {
  *c0 = (int)((long long)chunks * blockIdx.x / gridDim.x);
  *c1 = (int)((long long)chunks * (blockIdx.x + 1) / gridDim.x);
}

template <typename Table>
__global__ void __launch_bounds__(kThreads) clip_sum_kernel(const __grid_constant__ Table b, double* partial,
                                                            float keep) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ double part[kWarps];
  const int lane = threadIdx.x & 31;
  int c0, c1;
  run_of(b.chunks, &c0, &c1);
  // the run's end stays in L2, where the scaling begins
  const uint64_t pass = policy_pass(), hold = policy_keep();
  const int from = c1 - (int)(keep * (float)(c1 - c0));
  auto policy = [&](int c) { return c >= from ? hold : pass; };
  Squares squares;
  int c = c0 + (int)(threadIdx.x >> 5);
  if (c < c1) {
    int i = find_tensor(b, c);
    Piece p = piece_of(b.t[i], c);
    Held h0, h1;
    load_piece<0>(p, lane, h0, policy(c));
    while (c < c1) {
      const Piece now = p;
      load_piece<1>(now, lane, h1, policy(c));
      squares.add(now, h0);
      c += kWarps;
      if (c < c1) {
        while (i + 1 < b.n && c >= b.t[i + 1].chunk_begin) ++i;
        p = piece_of(b.t[i], c);
        load_piece<0>(p, lane, h0, policy(c));
      }
      squares.add(now, h1);
    }
  }
  const double sum = cta_sum<kWarps>(warp_total(squares, b, c0 + (int)(threadIdx.x >> 5), c1), part);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// This grid runs beside the one that writes `partial`, up to griddep_wait(): the pointer is not __restrict__, which would
// let the compiler read it earlier, or through a cache that does not see the writes.
template <typename Table>
__global__ void __launch_bounds__(32 * kScaleWarps)
    clip_scale_kernel(const __grid_constant__ Table b, const double* partial, int n_partial, float max_norm,
                      float* norm_out, float* coef_out) {
  __shared__ Coef s_coef;
  const int lane = threadIdx.x & 31;
  const uint64_t pass = policy_pass();
  int c0, c1;
  run_of(b.chunks, &c0, &c1);
  // the tensors were written before the first launch of the call began
  int c = c1 - 1 - (int)(threadIdx.x >> 5), i = 0;
  Piece p;
  Held h0, h1;
  if (c >= c0) {
    i = find_tensor(b, c);
    p = piece_of(b.t[i], c);
    load_piece<0>(p, lane, h0, pass);
  }
  griddep_wait();
  griddep_launch_dependents();
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int k = threadIdx.x; k < n_partial; k += 32) sum += __ldcg(partial + k);
    sum = warp_sum(sum);
    if (threadIdx.x == 0) s_coef = coef_of(sum, max_norm, norm_out, coef_out, blockIdx.x == 0);
  }
  __syncthreads();
  const Coef cf = s_coef;
  while (c >= c0) {
    const Piece now = p;
    load_piece<1>(now, lane, h1, pass);
    store_piece<0>(now, lane, h0, cf);
    c -= kScaleWarps;
    if (c >= c0) {
      while (c < b.t[i].chunk_begin) --i;
      p = piece_of(b.t[i], c);
      load_piece<0>(p, lane, h0, pass);
    }
    store_piece<1>(now, lane, h1, cf);
  }
}

template <typename Table>
__global__ void __launch_bounds__(32 * kOneWarps)
    clip_one_kernel(const __grid_constant__ Table b, float max_norm, float* norm_out, float* coef_out) {
  __shared__ double part[kOneWarps], all[kOneCtas];
  __shared__ Coef s_coef;
  const int lane = threadIdx.x & 31;
  // pieces go round the CTAs, so that few of them use every SM of the cluster
  const int c = (int)(threadIdx.x >> 5) * kOneCtas + (int)blockIdx.x;
  cluster_begun_arrive();
  griddep_wait();
  griddep_launch_dependents();
  Piece p;
  Held h0, h1;
  Squares squares;
  if (c < b.chunks) {
    p = piece_of(b.t[find_tensor(b, c)], c);
    load_piece<0>(p, lane, h0, policy_pass());
    load_piece<1>(p, lane, h1, policy_pass());
    squares.add(p, h0);
    squares.add(p, h1);
  }
  double sum = cta_sum<kOneWarps>(warp_total(squares, b, c, min(c + 1, b.chunks)), part);
  __syncwarp();
  cluster_begun_wait();
  if (threadIdx.x < kOneCtas) {
    sum = __shfl_sync((1u << kOneCtas) - 1u, sum, 0);
    const uint32_t to = mapa_shared(smem_u32(&all[blockIdx.x]), threadIdx.x);
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(sum) : "memory");
  }
  cluster_sync_all();
  if (threadIdx.x < 32) {
    double v = threadIdx.x < kOneCtas ? all[threadIdx.x] : 0.0;
    v = warp_sum(v);
    if (threadIdx.x == 0) s_coef = coef_of(v, max_norm, norm_out, coef_out, blockIdx.x == 0);
  }
  __syncthreads();
  if (c < b.chunks) {
    const Coef cf = s_coef;
    store_piece<0>(p, lane, h0, cf);
    store_piece<1>(p, lane, h1, cf);
  }
}

template <int N>
struct Table {
  ClipTensor t[N];
  int n, chunks;
};

// Lets `kernel` run in clusters of more than eight CTAs, once per device.
template <typename... KArgs>
cudaError_t allow_cluster_once(void (*kernel)(KArgs...), std::atomic<unsigned long long>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_acq_rel);
  return e;
}

// Runs fn with the batch as a table of the smallest capacity that holds it: the launch copies the whole argument.
template <typename Fn>
cudaError_t with_table(const ClipBatch& b, Fn fn) {
  auto sized = [&](auto& t) {
    for (int i = 0; i < b.n; ++i) t.t[i] = b.t[i];
    t.n = b.n;
    t.chunks = b.chunks;
    return fn(t);
  };
  if (b.n <= 16) {
    Table<16> t;
    return sized(t);
  }
  if (b.n <= 128) {
    Table<128> t;
    return sized(t);
  }
  if (b.n <= 448) {
    Table<448> t;
    return sized(t);
  }
  return fn(b);
}

}  // namespace

// One launch or two (us): 16384 elements 3.2 and 4.8, 131072 3.8 and 5.0, 245760 4.7 and 5.0; two pieces a warp, for
// twice the elements, took longer than two launches (524288: 7.9 and 5.3).
bool clip_is_small(const ClipBatch& b) { return b.chunks <= kOneCtas * kOneWarps; }

// A quarter of a CTA's warps at work are enough to keep its loads in flight; more CTAs cost more partial sums.
int clip_ctas(int chunks, int num_sms) {
  const int n = (chunks + kWarps / 4 - 1) / (kWarps / 4);
  return n < 1 ? 1 : n < num_sms ? n : num_sms;
}

cudaError_t launch_clip_sum(const ClipBatch& b, double* partial, int ctas, float keep, cudaStream_t st) {
  return with_table(b, [&](const auto& t) {
    return launch_kernel(clip_sum_kernel<std::decay_t<decltype(t)>>, dim3(ctas), dim3(kThreads), 0, st, 1, t, partial, keep);
  });
}

cudaError_t launch_clip_scale(const ClipBatch& b, const double* partial, int n_partial, float max_norm, float* norm,
                              float* coef, int ctas, cudaStream_t st) {
  return with_table(b, [&](const auto& t) {
    return launch_kernel(clip_scale_kernel<std::decay_t<decltype(t)>>, dim3(ctas), dim3(32 * kScaleWarps), 0, st, 1, t,
                         partial, n_partial, max_norm, norm, coef);
  });
}

cudaError_t launch_clip_one(const ClipBatch& b, float max_norm, float* norm, float* coef, cudaStream_t st) {
  return with_table(b, [&](const auto& t) {
    using T = std::decay_t<decltype(t)>;
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_cluster_once(clip_one_kernel<T>, done);
    if (e != cudaSuccess) return e;
    return launch_kernel(clip_one_kernel<T>, dim3(kOneCtas), dim3(32 * kOneWarps), 0, st, kOneCtas, t, max_norm, norm, coef);
  });
}

}  // namespace lora
