// Global norm of many gradient tensors, and their clipping to a bound:
//   norm = sqrt(sum g^2),  coef = norm > max_norm ? max_norm / norm : 1,  dst = coef * src
//
// A warp takes a piece of 1024 elements (4 KB of fp32) at a time, all its loads issued at once; the pieces are dealt
// to the warps in equal contiguous runs.  Small calls run as one launch, many tensors as two:
//   clip_one_kernel    one cluster, a piece per warp: the elements stay in registers between the sum and the scaling,
//                      the CTAs exchange their sums through distributed shared memory
//   clip_sum_kernel    the CTAs' sums of squares, one CTA per SM
//   clip_scale_kernel  every CTA adds these up again in the same order, then scales, from the last piece to the first:
//                      what was read last is still in L2
// All are bound by memory (a read for the norm, a read from L2 or HBM and a write for the scaling).  FP64 is scarce
// on this GPU (about 2 operations a clock and SM), so a lane's 32 squares are summed in fp32 and only that sum is
// added in fp64, and one warp per CTA adds the CTAs' sums.  The tensors' table is a kernel argument: no copy
// precedes the launches.
#include <type_traits>

#include "common.cuh"
#include "kernels.h"

namespace lora {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kOneCtas = 8;  // of the single cluster

// A piece's place: the elements before the first 16-byte boundary of src (head), the vectors behind them, the rest.
struct Piece {
  const ClipTensor* t;
  long long i0;  // first element
  int n, head, vecs;
};

__device__ __forceinline__ Piece piece_of(const ClipTensor& t, int c) {
  Piece p;
  p.t = &t;
  p.i0 = (long long)(c - t.chunk_begin) * kClipChunk;
  p.n = (int)min((long long)kClipChunk, t.n - p.i0);
  const int size = t.half ? 2 : 4, per = 16 / size;
  const uintptr_t a = reinterpret_cast<uintptr_t>(t.src) + (uintptr_t)p.i0 * size;
  p.head = min(p.n, (int)((16 - (a & 15)) & 15) / size);
  p.vecs = (p.n - p.head) / per;
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

constexpr int kVecs = kClipChunk / 4 / 32;  // 16-byte vectors of a lane (fp32; half of them with bf16)

// A lane's part of a piece: vectors lane, lane + 32, ..; one element of the head or of the rest.
struct Held {
  uint4 v[kVecs];
  float edge;
};

__device__ __forceinline__ int edge_index(const Piece& p, int lane) {
  const int body = p.head + p.vecs * (p.t->half ? 8 : 4), i = lane < p.head ? lane : body + lane - p.head;
  return i < p.n && (lane < p.head || i >= body) ? i : -1;
}

__device__ __forceinline__ void load_piece(const Piece& p, int lane, Held& h) {
  const int size = p.t->half ? 2 : 4;
  const uint8_t* src = static_cast<const uint8_t*>(p.t->src) + p.i0 * size;
  const uint4* v = reinterpret_cast<const uint4*>(src + p.head * size);
#pragma unroll
  for (int q = 0; q < kVecs; ++q)
    h.v[q] = lane + 32 * q < p.vecs ? v[lane + 32 * q] : make_uint4(0u, 0u, 0u, 0u);
  const int e = edge_index(p, lane);
  h.edge = e < 0 ? 0.f
                 : (p.t->half ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(src)[e])
                              : reinterpret_cast<const float*>(src)[e]);
}

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Sum of (scale x)^2 over the lane's elements.
__device__ __forceinline__ float squares(const Held& h, bool half, float scale) {
  float s[4] = {h.edge * scale * (h.edge * scale), 0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < kVecs; ++q) {
    const uint32_t w[4] = {h.v[q].x, h.v[q].y, h.v[q].z, h.v[q].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (half) {
        const float a = lo_bf16(w[e]) * scale, b = hi_bf16(w[e]) * scale;
        s[e] = fmaf(a, a, s[e]);
        s[e] = fmaf(b, b, s[e]);
      } else {
        const float a = __uint_as_float(w[e]) * scale;
        s[e] = fmaf(a, a, s[e]);
      }
    }
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// The same in fp64 range: a sum that fp32 may have lost squares of (below 2^-60, or beyond 2^100) is formed again
// from scaled elements.  2^60 twice brings the smallest subnormal's square into range; 2^-80 the largest element's.
__device__ __forceinline__ double sum_squares(const Held& h, bool half) {
  float s = squares(h, half, 1.f);
  double unit = 1.0;
  if (s < 0x1p-60f) {
    s = squares(h, half, 0x1p60f);
    unit = 0x1p-120;
    if (s < 0x1p-60f) {
      s = squares(h, half, 0x1p120f);
      unit = 0x1p-240;
    }
  } else if (!(s <= 0x1p100f)) {
    s = squares(h, half, 0x1p-80f);
    unit = 0x1p160;
  }
  return (double)s * unit;
}

struct Coef {
  float coef, pre, mul;
};

// A norm that is not finite (an infinity or a NaN in a gradient) leaves the tensors as they are.  A coefficient that
// fp32 would round as a subnormal is applied in two factors.
__device__ __forceinline__ Coef coef_of(double total, float max_norm, float* norm_out, float* coef_out, bool writes) {
  const double norm = sqrt(total);
  const double exact = isfinite(norm) && norm > (double)max_norm ? (double)max_norm / norm : 1.0;
  Coef c;
  c.coef = (float)exact;
  c.pre = exact < 0x1p-100 ? 0x1p-64f : 1.f;
  c.mul = (float)(exact * (exact < 0x1p-100 ? 0x1p64 : 1.0));
  if (writes) {
    *norm_out = (float)norm;
    if (coef_out) *coef_out = c.coef;
  }
  return c;
}

__device__ __forceinline__ void store_piece(const Piece& p, int lane, const Held& h, const Coef& c) {
  const ClipTensor& t = *p.t;
  const bool copy = c.coef == 1.f;  // also keeps a NaN's bits
  if (!t.dst || (copy && t.dst == t.src)) return;
  const int size = t.half ? 2 : 4;
  uint8_t* dst = static_cast<uint8_t*>(t.dst) + p.i0 * size;
  uint8_t* body = dst + p.head * size;
  const bool whole = (reinterpret_cast<uintptr_t>(body) & 15) == 0;
#pragma unroll
  for (int q = 0; q < kVecs; ++q) {
    const int i = lane + 32 * q;
    if (i >= p.vecs) break;
    uint32_t w[4] = {h.v[q].x, h.v[q].y, h.v[q].z, h.v[q].w};
    if (!copy) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = t.half ? pack_bf16x2(lo_bf16(w[e]) * c.pre * c.mul, hi_bf16(w[e]) * c.pre * c.mul)
                      : __float_as_uint(__uint_as_float(w[e]) * c.pre * c.mul);
    }
    if (whole) {
      __stcs(reinterpret_cast<uint4*>(body) + i, make_uint4(w[0], w[1], w[2], w[3]));
    } else if (t.half) {  // the destination lies differently from the source
      uint16_t* o = reinterpret_cast<uint16_t*>(body) + 8 * i;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[2 * e] = (uint16_t)w[e];
        o[2 * e + 1] = (uint16_t)(w[e] >> 16);
      }
    } else {
      uint32_t* o = reinterpret_cast<uint32_t*>(body) + 4 * i;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = w[e];
    }
  }
  const int e = edge_index(p, lane);
  if (e < 0) return;
  const float v = copy ? h.edge : h.edge * c.pre * c.mul;
  if (t.half)
    reinterpret_cast<__nv_bfloat16*>(dst)[e] = copy ? static_cast<const __nv_bfloat16*>(t.src)[p.i0 + e]
                                                    : __float2bfloat16(v);
  else
    reinterpret_cast<float*>(dst)[e] = v;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Warps' sums added by warp 0 (valid there); one barrier.
__device__ __forceinline__ double cta_sum(double v, double* part) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  return threadIdx.x < 32 ? warp_sum(part[threadIdx.x]) : 0.0;
}

template <typename Table>
__global__ void __launch_bounds__(kThreads) clip_sum_kernel(const __grid_constant__ Table b,
                                                            double* __restrict__ partial) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ double part[kWarps];
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * kWarps, w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int c0 = (int)(b.chunks * w / warps), c1 = (int)(b.chunks * (w + 1) / warps);
  double sum = 0.0;
  int i = c0 < c1 ? find_tensor(b, c0) : 0;
  for (int c = c0; c < c1; ++c) {
    while (i + 1 < b.n && c >= b.t[i + 1].chunk_begin) ++i;
    Held h;
    load_piece(piece_of(b.t[i], c), lane, h);
    sum += sum_squares(h, b.t[i].half);
  }
  sum = cta_sum(sum, part);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <typename Table>
__global__ void __launch_bounds__(kThreads) clip_scale_kernel(const __grid_constant__ Table b,
                                                              const double* __restrict__ partial, int n_partial,
                                                              float max_norm, float* __restrict__ norm_out,
                                                              float* __restrict__ coef_out) {
  __shared__ Coef s_coef;
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * kWarps, w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int c0 = (int)(b.chunks * w / warps), c1 = (int)(b.chunks * (w + 1) / warps);
  int i = c0 < c1 ? find_tensor(b, c1 - 1) : 0;
  griddep_wait();
  griddep_launch_dependents();
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int k = threadIdx.x; k < n_partial; k += 32) sum += partial[k];
    sum = warp_sum(sum);
    if (threadIdx.x == 0) s_coef = coef_of(sum, max_norm, norm_out, coef_out, blockIdx.x == 0);
  }
  __syncthreads();
  const Coef cf = s_coef;
  for (int c = c1 - 1; c >= c0; --c) {
    while (c < b.t[i].chunk_begin) --i;
    const Piece p = piece_of(b.t[i], c);
    Held h;
    load_piece(p, lane, h);
    store_piece(p, lane, h, cf);
  }
}

template <typename Table>
__global__ void __launch_bounds__(kThreads) clip_one_kernel(const __grid_constant__ Table b, float max_norm,
                                                            float* __restrict__ norm_out,
                                                            float* __restrict__ coef_out) {
  __shared__ double part[kWarps], all[kOneCtas];
  __shared__ Coef s_coef;
  const int lane = threadIdx.x & 31;
  // pieces go round the CTAs, so that few of them use every SM of the cluster
  const int c = (int)(threadIdx.x >> 5) * kOneCtas + (int)blockIdx.x;
  griddep_wait();
  griddep_launch_dependents();
  Piece p;
  Held h;
  double sum = 0.0;
  if (c < b.chunks) {
    const ClipTensor& t = b.t[find_tensor(b, c)];
    p = piece_of(t, c);
    load_piece(p, lane, h);
    sum = sum_squares(h, t.half);
  }
  sum = cta_sum(sum, part);
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
  if (c < b.chunks) store_piece(p, lane, h, s_coef);
}

template <int N>
struct Table {
  ClipTensor t[N];
  int n, chunks;
};

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
  return fn(b);
}

}  // namespace

bool clip_is_small(const ClipBatch& b) { return b.chunks <= kOneCtas * kWarps; }

// A quarter of a CTA's warps at work are enough to keep its loads in flight; more CTAs cost more partial sums.
int clip_ctas(int chunks, int num_sms) {
  const int n = (chunks + kWarps / 4 - 1) / (kWarps / 4);
  return n < 1 ? 1 : n < num_sms ? n : num_sms;
}

cudaError_t launch_clip_sum(const ClipBatch& b, double* partial, int ctas, cudaStream_t st) {
  return with_table(b, [&](const auto& t) {
    return launch_kernel(clip_sum_kernel<std::decay_t<decltype(t)>>, dim3(ctas), dim3(kThreads), 0, st, 1, t, partial);
  });
}

cudaError_t launch_clip_scale(const ClipBatch& b, const double* partial, int n_partial, float max_norm, float* norm,
                              float* coef, int ctas, cudaStream_t st) {
  return with_table(b, [&](const auto& t) {
    return launch_kernel(clip_scale_kernel<std::decay_t<decltype(t)>>, dim3(ctas), dim3(kThreads), 0, st, 1, t,
                         partial, n_partial, max_norm, norm, coef);
  });
}

cudaError_t launch_clip_one(const ClipBatch& b, float max_norm, float* norm, float* coef, cudaStream_t st) {
  return with_table(b, [&](const auto& t) {
    return launch_kernel(clip_one_kernel<std::decay_t<decltype(t)>>, dim3(kOneCtas), dim3(kThreads), 0, st, kOneCtas,
                         t, max_norm, norm, coef);
  });
}

}  // namespace lora
