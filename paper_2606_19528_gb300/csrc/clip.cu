// Global norm of many gradient tensors, and their clipping to a bound:
//   norm = sqrt(sum g^2),  coef = norm > max_norm ? max_norm / norm : 1,  dst = coef * src
//
// A warp takes a piece of 512 elements (2 KB of fp32) at a time, the next one's loads issued before it is used; the
// pieces are dealt to the CTAs in equal contiguous runs.  Small calls run as one launch, many tensors as two:
//   clip_one_kernel    one cluster, two pieces per warp: the elements stay in registers between the sum and the
//                      scaling, the CTAs exchange their sums through distributed shared memory
//   clip_sum_kernel    the CTAs' sums of squares, one CTA per SM
//   clip_scale_kernel  every CTA adds these up again in the same order, then scales, from the last piece to the first:
//                      what was read last is still in L2
// All are bound by memory (a read for the norm, a read from L2 or HBM and a write for the scaling).  FP64 is scarce
// on this GPU (about 2 operations a clock and SM), so a lane's 16 squares are summed in fp32 and these sums as pairs
// of fp32; only the warps' sums are added in fp64.  The tensors' table is a kernel argument: no copy precedes the
// launches.
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "pair.cuh"

namespace lora {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kOneCtas = 8, kOnePieces = 2;  // of the single cluster; a warp's pieces in it

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

constexpr int kVecs = kClipChunk / 4 / 32;  // 16-byte vectors of a lane (fp32; half of them with bf16)

// A lane's part of a piece: vectors lane, lane + 32, ..; one element of the head or of the rest.
struct Held {
  uint4 v[kVecs];
  uint32_t edge;  // as fp32
};

// The element of the head or the rest that a lane holds, or -1.
__device__ __forceinline__ int edge_index(const Piece& p, int lane) {
  const int body = p.vecs << (p.half ? 3 : 2), i = lane < p.head ? lane : body + lane;
  return i < p.n ? i : -1;
}

__device__ __forceinline__ void load_piece(const Piece& p, int lane, Held& h) {
  const uint4* v = reinterpret_cast<const uint4*>(p.src + (p.head << (p.half ? 1 : 2)));
#pragma unroll
  for (int q = 0; q < kVecs; ++q)
    h.v[q] = lane + 32 * q < p.vecs ? v[lane + 32 * q] : make_uint4(0u, 0u, 0u, 0u);
  const int e = edge_index(p, lane);
  h.edge = 0u;
  if (e >= 0)
    h.edge = p.half ? (uint32_t) reinterpret_cast<const uint16_t*>(p.src)[e] << 16
                    : reinterpret_cast<const uint32_t*>(p.src)[e];
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
  for (int q = 0; q < (HALF ? kVecs / 2 : kVecs); ++q) {
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

// The same of a piece that is loaded again, for the rare sums that need it.
__device__ __noinline__ float squares_scaled(const uint8_t* src, int n, int head, int vecs, bool half, float scale) {
  Piece p;
  p.src = src;
  p.n = n;
  p.head = head;
  p.vecs = vecs;
  p.half = half;
  Held h;
  load_piece(p, threadIdx.x & 31, h);
  return half ? squares<true, true>(h, scale) : squares<false, true>(h, scale);
}

// A lane's sum of squares: `most` holds those that fp32 forms without loss, `rest` what it cannot (below 2^-60, where
// squares may have been lost, or beyond 2^100), from elements scaled by a power of two: 2^60 twice brings the
// smallest subnormal's square into range, 2^-80 the largest element's.
struct Squares {
  Pair most{};
  double rest = 0.0;
  __device__ __forceinline__ void add(const Piece& p, const Held& h) {
    float s = p.half ? squares<true, false>(h, 1.f) : squares<false, false>(h, 1.f);
    if (s >= 0x1p-60f && s <= 0x1p100f) {
      most.add(s);
      return;
    }
    double unit = 0x1p160;
    if (s < 0x1p-60f) {
      s = squares_scaled(p.src, p.n, p.head, p.vecs, p.half, 0x1p60f);
      unit = 0x1p-120;
      if (s < 0x1p-60f) {
        s = squares_scaled(p.src, p.n, p.head, p.vecs, p.half, 0x1p120f);
        unit = 0x1p-240;
      }
      if (s == 0.f) return;
    } else {
      s = squares_scaled(p.src, p.n, p.head, p.vecs, p.half, 0x1p-80f);
    }
    rest += (double)s * unit;
  }
  // over the warp's lanes
  __device__ __forceinline__ double total() const {
    double v = warp_sum(most).wide();
    if (__any_sync(0xffffffffu, rest != 0.0)) v += warp_sum(rest);
    return v;
  }
};

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

template <bool HALF>
__device__ __forceinline__ void store_scaled(const Piece& p, int lane, const Held& h, const Coef& c) {
  const bool copy = c.coef == 1.f;  // also keeps a NaN's bits
  auto scaled = [&](float x) { return x * c.pre * c.mul; };
  uint8_t* body = p.dst + (p.head << (HALF ? 1 : 2));
  const bool whole = (reinterpret_cast<uintptr_t>(body) & 15) == 0;
#pragma unroll
  for (int q = 0; q < (HALF ? kVecs / 2 : kVecs); ++q) {
    const int i = lane + 32 * q;
    uint32_t w[4] = {h.v[q].x, h.v[q].y, h.v[q].z, h.v[q].w};
    if (!copy) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = HALF ? pack_bf16x2(scaled(lo_bf16(w[e])), scaled(hi_bf16(w[e])))
                    : __float_as_uint(scaled(__uint_as_float(w[e])));
    }
    if (i >= p.vecs) continue;
    if (whole) {
      __stcs(reinterpret_cast<uint4*>(body) + i, make_uint4(w[0], w[1], w[2], w[3]));
    } else if (HALF) {  // the destination lies differently from the source
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
  const float x = __uint_as_float(h.edge);
  if (HALF)
    reinterpret_cast<uint16_t*>(p.dst)[e] =
        copy ? (uint16_t)(h.edge >> 16) : __bfloat16_as_ushort(__float2bfloat16(scaled(x)));
  else
    reinterpret_cast<float*>(p.dst)[e] = copy ? x : scaled(x);
}

__device__ __forceinline__ void store_piece(const Piece& p, int lane, const Held& h, const Coef& c) {
  if (!p.dst || (c.coef == 1.f && p.same)) return;
  if (p.half)
    store_scaled<true>(p, lane, h, c);
  else
    store_scaled<false>(p, lane, h, c);
}

// The CTA's sum, in warp 0; one barrier.
__device__ __forceinline__ double cta_sum(const Squares& s, double* part) {
  const double v = s.total();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  return threadIdx.x < 32 ? warp_sum(part[threadIdx.x]) : 0.0;
}

// The run of pieces [c0, c1) that is this CTA's; its warps take them in turn.
__device__ __forceinline__ void run_of(int chunks, int* c0, int* c1) {
  *c0 = (int)((long long)chunks * blockIdx.x / gridDim.x);
  *c1 = (int)((long long)chunks * (blockIdx.x + 1) / gridDim.x);
}

template <typename Table>
__global__ void __launch_bounds__(kThreads) clip_sum_kernel(const __grid_constant__ Table b,
                                                            double* __restrict__ partial) {
  griddep_wait();
  griddep_launch_dependents();
  __shared__ double part[kWarps];
  const int lane = threadIdx.x & 31;
  int c0, c1;
  run_of(b.chunks, &c0, &c1);
  Squares squares;
  int c = c0 + (int)(threadIdx.x >> 5);
  if (c < c1) {
    int i = find_tensor(b, c);
    Piece p = piece_of(b.t[i], c);
    Held h;
    load_piece(p, lane, h);
    while (c < c1) {
      c += kWarps;
      Piece next_p = p;
      Held next;
      if (c < c1) {
        while (i + 1 < b.n && c >= b.t[i + 1].chunk_begin) ++i;
        next_p = piece_of(b.t[i], c);
        load_piece(next_p, lane, next);
      }
      squares.add(p, h);
      p = next_p;
      h = next;
    }
  }
  const double sum = cta_sum(squares, part);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <typename Table>
__global__ void __launch_bounds__(kThreads) clip_scale_kernel(const __grid_constant__ Table b,
                                                              const double* __restrict__ partial, int n_partial,
                                                              float max_norm, float* __restrict__ norm_out,
                                                              float* __restrict__ coef_out) {
  __shared__ Coef s_coef;
  const int lane = threadIdx.x & 31;
  int c0, c1;
  run_of(b.chunks, &c0, &c1);
  // the tensors were written before the first launch of the call began
  int c = c1 - 1 - (int)(threadIdx.x >> 5), i = 0;
  Piece p;
  Held h;
  if (c >= c0) {
    i = find_tensor(b, c);
    p = piece_of(b.t[i], c);
    load_piece(p, lane, h);
  }
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
  while (c >= c0) {
    c -= kWarps;
    Piece next_p = p;
    Held next;
    if (c >= c0) {
      while (c < b.t[i].chunk_begin) --i;
      next_p = piece_of(b.t[i], c);
      load_piece(next_p, lane, next);
    }
    store_piece(p, lane, h, cf);
    p = next_p;
    h = next;
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
  const int c0 = (int)(threadIdx.x >> 5) * kOneCtas + (int)blockIdx.x;
  griddep_wait();
  griddep_launch_dependents();
  Piece p[kOnePieces];
  Held h[kOnePieces];
#pragma unroll
  for (int k = 0; k < kOnePieces; ++k) {
    const int c = c0 + k * kOneCtas * kWarps;
    if (c < b.chunks) {
      p[k] = piece_of(b.t[find_tensor(b, c)], c);
      load_piece(p[k], lane, h[k]);
    }
  }
  Squares squares;
#pragma unroll
  for (int k = 0; k < kOnePieces; ++k)
    if (c0 + k * kOneCtas * kWarps < b.chunks) squares.add(p[k], h[k]);
  double sum = cta_sum(squares, part);
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
#pragma unroll
  for (int k = 0; k < kOnePieces; ++k)
    if (c0 + k * kOneCtas * kWarps < b.chunks) store_piece(p[k], lane, h[k], s_coef);
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

bool clip_is_small(const ClipBatch& b) { return b.chunks <= kOneCtas * kWarps * kOnePieces; }

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
