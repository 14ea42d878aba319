// Forward of adapted projections with 4-bit weights for 1 to 16 tokens:
//   su = scale * x A^T          one block per adapter row (fp32, not rounded)
//   y  = x W^T + su B^T         W[n, k] = bf16(s q + b) from its 4-bit codes
//
// With so few tokens every weight is used once or a handful of times, so the call is bound by reading 9/16 byte per
// weight.  A weight is still dequantized (2 FMAs and about 1.75 integer operations per pair) and multiplied; the
// products go through mma.sync m16n8k16, whose 8 columns are the tokens: an accumulation on the FMA units would
// take two conversions and 2 T FMAs per pair more.  (The tcgen05 path needs its operands in shared memory: the
// round trip of the dequantized weights costs more than the products of 16 tokens.)
#include "common.cuh"
#include "kernels.h"

namespace lora {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kTileN = 16;  // output rows of a tile: M of the MMA

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float2 bf2(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

// One block per (projection, adapter row j): su[t, j] = scale * x_t . A_j.
constexpr int kSuThreads = 128;
__global__ void __launch_bounds__(kSuThreads) decode_su_kernel(const __grid_constant__ DecodeBatch b) {
  griddep_wait();
  griddep_launch_dependents();
  int i = 0;
  while (i + 1 < b.n && (int)blockIdx.x >= b.p[i + 1].row_begin) ++i;
  const DecodeProj& p = b.p[i];
  const int j = (int)blockIdx.x - p.row_begin, vecs = p.K / 8;
  const uint4* a4 = reinterpret_cast<const uint4*>(p.A + (long long)j * p.K);
  float acc[kDecodeMaxT];
#pragma unroll
  for (int t = 0; t < kDecodeMaxT; ++t) acc[t] = 0.f;
  for (int v = threadIdx.x; v < vecs; v += kSuThreads) {
    const uint4 a = a4[v];
    const uint32_t aw[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int t = 0; t < kDecodeMaxT; ++t) {
      if (t < p.T) {
        const uint4 x = reinterpret_cast<const uint4*>(p.x + (long long)t * p.K)[v];
        const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float2 fa = bf2(aw[q]), fx = bf2(xw[q]);
          acc[t] = fmaf(fa.x, fx.x, acc[t]);
          acc[t] = fmaf(fa.y, fx.y, acc[t]);
        }
      }
    }
  }
  __shared__ float part[kSuThreads / 32][kDecodeMaxT];
#pragma unroll
  for (int t = 0; t < kDecodeMaxT; ++t) {
    float v = acc[t];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5][t] = v;
  }
  __syncthreads();
  if ((int)threadIdx.x < p.T) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kSuThreads / 32; ++w) v += part[w][threadIdx.x];
    p.su[threadIdx.x * p.r + j] = p.scale * v;
  }
}

// One block per 16 output rows.  Each warp takes every eighth chunk of 128 columns; lane (g, t) of it holds the 32
// columns 32 t .. of rows g and g + 8: a word of 8 codes makes the fragments of two MMAs, whose k index is then a
// permutation of the columns that the activation's fragments share (16 consecutive bytes of token g).
template <int NT>  // tokens / 8
__global__ void __launch_bounds__(kThreads) decode_kernel(const __grid_constant__ DecodeBatch b) {
  if (b.rows == 0) griddep_wait();  // the launch before is not this call's
  griddep_launch_dependents();
  int i = 0;
  while (i + 1 < b.n && (int)blockIdx.x >= b.p[i + 1].tile_begin) ++i;
  const DecodeProj& p = b.p[i];
  const int n0 = ((int)blockIdx.x - p.tile_begin) * kTileN;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int K = p.K;
  const long long r0 = min(n0 + g, p.N - 1), r1 = min(n0 + g + 8, p.N - 1);
  const uint8_t *c0 = p.codes + r0 * (K / 2), *c1 = p.codes + r1 * (K / 2);
  const uint32_t* q0 = reinterpret_cast<const uint32_t*>(p.params) + r0 * (K / 64);
  const uint32_t* q1 = reinterpret_cast<const uint32_t*>(p.params) + r1 * (K / 64);
  float acc[NT][4];
#pragma unroll
  for (int m = 0; m < NT; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[m][e] = 0.f;
  for (int k0 = 128 * warp; k0 < K; k0 += 128 * kWarps) {
    const int k = k0 + 32 * t;
    const bool in = k < K;  // K is a multiple of 64: the last chunk may be half a one
    uint4 w0 = make_uint4(0u, 0u, 0u, 0u), w1 = w0;
    uint32_t s0 = 0, s1 = 0;
    uint4 xv[NT][4];
    if (in) {
      w0 = __ldcs(reinterpret_cast<const uint4*>(c0 + k / 2));
      w1 = __ldcs(reinterpret_cast<const uint4*>(c1 + k / 2));
      s0 = q0[k / 64];
      s1 = q1[k / 64];
    }
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const int tok = g + 8 * m;
      const uint4* xp = reinterpret_cast<const uint4*>(p.x + (long long)tok * K + k);
#pragma unroll
      for (int q = 0; q < 4; ++q) xv[m][q] = in && tok < p.T ? xp[q] : make_uint4(0u, 0u, 0u, 0u);
    }
    const uint32_t sa = __byte_perm(s0, 0u, 0x1010), ba = __byte_perm(s0, 0u, 0x3232);
    const uint32_t sb = __byte_perm(s1, 0u, 0x1010), bb = __byte_perm(s1, 0u, 0x3232);
    const uint32_t u0[4] = {w0.x, w0.y, w0.z, w0.w}, u1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t a0 = dq_pair(u0[q] >> (8 * h), sa, ba), a1 = dq_pair(u1[q] >> (8 * h), sb, bb);
        const uint32_t a2 = dq_pair(u0[q] >> (8 * h + 4), sa, ba), a3 = dq_pair(u1[q] >> (8 * h + 4), sb, bb);
#pragma unroll
        for (int m = 0; m < NT; ++m)
          mma_bf16(acc[m], a0, a1, a2, a3, h ? xv[m][q].z : xv[m][q].x, h ? xv[m][q].w : xv[m][q].y);
      }
    }
  }
  __shared__ float red[kWarps][NT * 8][kTileN + 1];
#pragma unroll
  for (int m = 0; m < NT; ++m) {
    red[warp][8 * m + 2 * t][g] = acc[m][0];
    red[warp][8 * m + 2 * t + 1][g] = acc[m][1];
    red[warp][8 * m + 2 * t][g + 8] = acc[m][2];
    red[warp][8 * m + 2 * t + 1][g + 8] = acc[m][3];
  }
  __syncthreads();
  if (b.rows) griddep_wait();  // su
  const int tok = threadIdx.x / kTileN, n = n0 + (int)threadIdx.x % kTileN;
  if (tok < p.T && n < p.N) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += red[w][tok][n - n0];
    float u = 0.f;
    const float* su = p.su + tok * p.r;
    const __nv_bfloat16* B = p.B + (long long)n * p.r;
    for (int j = 0; j < p.r; ++j) u = fmaf(su[j], __bfloat162float(B[j]), u);
    p.y[(long long)tok * p.N + n] = __float2bfloat16(v + u);
  }
}

}  // namespace

cudaError_t launch_decode(DecodeBatch& b, int num_sms, cudaStream_t st) {
  (void)num_sms;
  b.tiles = b.rows = 0;
  int most = 1;
  for (int i = 0; i < b.n; ++i) {
    DecodeProj& p = b.p[i];
    p.tile_begin = b.tiles;
    p.row_begin = b.rows;
    b.tiles += (p.N + kTileN - 1) / kTileN;
    b.rows += p.r;
    if (p.T > most) most = p.T;
  }
  if (b.rows) {
    const cudaError_t e = launch_kernel(decode_su_kernel, dim3(b.rows), dim3(kSuThreads), 0, st, 1, b);
    if (e != cudaSuccess) return e;
  }
  return most <= 8 ? launch_kernel(decode_kernel<1>, dim3(b.tiles), dim3(kThreads), 0, st, 1, b)
                   : launch_kernel(decode_kernel<2>, dim3(b.tiles), dim3(kThreads), 0, st, 1, b);
}

}  // namespace lora
