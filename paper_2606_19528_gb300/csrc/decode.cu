// Forward of adapted projections with 4-bit weights for 1 to 16 tokens:
//   decode_su_kernel    su = scale * x A^T, one block per adapter row
//   decode_kernel       y  = x W^T + su B^T, W[n, k] = bf16(s q + b) from its 4-bit codes, 16 rows of W per block
//   decode_wide_kernel  the same, for many rows (decode_wide.cu)
//
// With so few tokens every weight is used once or a handful of times, so the call is bound by reading 9/16 byte per
// weight, and next by the instructions that dequantize it; small calls are bound by a chain of latencies (launch,
// codes, products, the warps' sums) and by the host's launches.  Dequantizing takes 9 instructions per 8 codes
// (dq40_word); the sums are scaled back by 2^40.  The products go through mma.sync m16n8k16, whose 8 columns are the
// tokens: on the FMA units a pair of weights would take two conversions and 2 T FMAs more.  An MMA holds a sub-core's
// tensor unit for 24 clocks, which bounds 9 to 16 tokens; the wide launch goes past that.
//
// su enters the same MMAs as three bf16 terms, which hold all 24 bits of its fp32 value: rounding it to bf16 would
// add an error of 2^-9 of the adapter's part.
//
// One token, q, k and v of 3072 columns (N 3072, 1024, 1024; r 16), 9.3 MB: 5.4 us, 1.7 TB/s; 8192 x 3072: 7.2 us, 2
// TB/s; five tokens, two of 2048 x 11008, r 64, 29 MB: 10.8 us, 2.7 TB/s.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace lora {
namespace {

constexpr int kTileN = 16;       // output rows of a tile: M of the MMA
constexpr int kChunk = 128;      // columns of a warp's step: two 64-wide groups, 32 columns a lane
constexpr int kMostThreads = 512;
constexpr int kRedPitch = 20;    // floats: the partial sums' stores meet no bank twice

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint4 load_codes(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Where column `col` of token `tok` lies, in 16-bit units.
__device__ __forceinline__ int su_at(int r, int tok, int col, int term) {
  const int c = col & 15;
  return 2 * ((tok * su_steps(r) + col / 16) * kSuWords + (c & 7) / 2 * 8 + c / 8 * 4 + term) + (c & 1);
}
__device__ __forceinline__ int su_image_at(int r, int tok, int col, int term) {
  return (term * su_blocks(r) + col / 64) * (kSuBlock / 2) + tok * 64 + ((col % 64 / 8) ^ (tok & 7)) * 8 + col % 8;
}

// One block per (projection, adapter row j): su[t, j] = scale * x_t . A_j for up to TT tokens.
constexpr int kSuThreads = 256;
template <int TT, typename Table>
__global__ void __launch_bounds__(kSuThreads) decode_su_kernel(const __grid_constant__ Table b) {
  griddep_wait();
  griddep_launch_dependents();
  int i = 0;
  while (i + 1 < b.n && (int)blockIdx.x >= b.p[i + 1].row_begin) ++i;
  const DecodeProj& p = b.p[i];
  const int j = (int)blockIdx.x - p.row_begin, vecs = p.K / 8;
  const uint4* a4 = reinterpret_cast<const uint4*>(p.A + (long long)j * p.K);
  float acc[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[t] = 0.f;
  for (int v = threadIdx.x; v < vecs; v += kSuThreads) {
    const uint4 a = a4[v];
    uint4 x[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) x[t] = reinterpret_cast<const uint4*>(p.x + (long long)min(t, p.T - 1) * p.K)[v];
    const uint32_t aw[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const uint32_t xw[4] = {x[t].x, x[t].y, x[t].z, x[t].w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        acc[t] = fmaf(lo_bf16(aw[q]), lo_bf16(xw[q]), acc[t]);
        acc[t] = fmaf(hi_bf16(aw[q]), hi_bf16(xw[q]), acc[t]);
      }
    }
  }
  __shared__ float part[kSuThreads / 32][TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
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
    v *= p.scale * 0x1p-40f;
    __nv_bfloat16 *su = reinterpret_cast<__nv_bfloat16*>(p.su), *image = reinterpret_cast<__nv_bfloat16*>(p.su_image);
    auto put = [&](int col, int e, __nv_bfloat16 term) {
      su[su_at(p.r, threadIdx.x, col, e)] = term;
      image[su_image_at(p.r, threadIdx.x, col, e)] = term;
    };
#pragma unroll
    for (int e = 0; e < kSuTerms; ++e) {
      const __nv_bfloat16 term = __float2bfloat16(v);
      put(j, e, term);
      v = isfinite(v) ? v - __bfloat162float(term) : 0.f;
    }
    if (j == p.r - 1)
      for (int col = p.r; col < 16 * su_steps(p.r); ++col)
        for (int e = 0; e < kSuTerms; ++e) put(col, e, __float2bfloat16(0.f));
  }
}

// What a warp reads per step of 128 columns: 32 codes of row g and of row g + 8 for each lane (g, t), with their (s, b).
struct Step {
  uint4 w0, w1;
  uint32_t s0, s1;
};

// One block per 16 output rows, its warps sharing out the columns: warp i has every warps-th chunk of 128 from i on, and
// every warps-th 16 of the adapter's columns.  A step's weights are loaded while the one before is computed; loading
// two to four steps ahead takes the registers of as many warps and is slower.  A lane's word of 8 codes makes the
// fragments of two MMAs, whose k index is then a permutation of the columns; the activation's fragments share it: 16
// consecutive bytes of token g, which come through L1.  Activations and adapters are read by plain loads, since a launch
// that this one overlaps may have written them; codes and parameters, which do not change, are not.
//
// OWN: each block computes su of its projection beside y, from all of A, in the same loop: 16 adapter rows are one more
// tile, whose fragments come from A as they lie; no launch goes before.
template <int NT, bool OWN, typename Table>  // tokens / 8
__global__ void __launch_bounds__(kMostThreads) decode_kernel(const __grid_constant__ Table b) {
  constexpr int kChains = NT == 1 ? 2 : 1;  // of dependent MMAs: two at least
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  if (!b.after_su) griddep_wait();  // otherwise the launch before is this call's, and began after its inputs were there
  griddep_launch_dependents();
  int i = 0;
  while (i + 1 < b.n && (int)blockIdx.x >= b.p[i + 1].tile_begin) ++i;
  const DecodeProj& p = b.p[i];
  const int n0 = ((int)blockIdx.x - p.tile_begin) * kTileN, K = p.K, T = p.T, r = p.r;
  const long long r0 = min(n0 + g, p.N - 1), r1 = min(n0 + g + 8, p.N - 1);
  const uint8_t *c0 = p.codes + r0 * (K / 2) + 16 * t, *c1 = p.codes + r1 * (K / 2) + 16 * t;
  const uint32_t* q0 = reinterpret_cast<const uint32_t*>(p.params) + r0 * (K / 64) + t / 2;
  const uint32_t* q1 = reinterpret_cast<const uint32_t*>(p.params) + r1 * (K / 64) + t / 2;
  // K is a multiple of 64: the last chunk may be half a one, where s = b = 0 make the weights zero
  auto fetch = [&](Step& s, int c) {
    s.s0 = s.s1 = 0u;
    s.w0 = s.w1 = make_uint4(0u, 0u, 0u, 0u);
    if (c * kChunk + 32 * t < K) {
      s.w0 = load_codes(c0 + c * (kChunk / 2));
      s.w1 = load_codes(c1 + c * (kChunk / 2));
      s.s0 = __ldg(q0 + 2 * c);
      s.s1 = __ldg(q1 + 2 * c);
    }
  };
  Step s;
  fetch(s, warp);

  // the adapter's A operand of 16 columns: rows g and g + 8 of B, columns 2 t (+ 1) and 2 t + 8 (+ 9)
  auto load_adapter = [&](int j0, uint32_t (&a)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int n = n0 + g + 8 * (e & 1), j = j0 + 2 * t + 8 * (e >> 1);
      const uint16_t* q = reinterpret_cast<const uint16_t*>(p.B) + (long long)n * r + j;
      a[e] = 0u;
      if (n < p.N && j < r) {
        if (r % 2 == 0)
          a[e] = *reinterpret_cast<const uint32_t*>(q);
        else
          a[e] = q[0] | (j + 1 < r ? (uint32_t)q[1] << 16 : 0u);
      }
    }
  };
  uint32_t adapter[4];
  load_adapter(16 * warp, adapter);

  float acc[kChains][NT][4] = {}, sacc[OWN ? NT : 1][4] = {};
  const uint4 *a0 = nullptr, *a1 = nullptr;
  if (OWN && r) {
    a0 = reinterpret_cast<const uint4*>(p.A + (long long)min(g, r - 1) * K + 32 * t);
    a1 = reinterpret_cast<const uint4*>(p.A + (long long)min(g + 8, r - 1) * K + 32 * t);
  }
  const uint4* x4[NT];  // columns past T are dropped: whatever token their fragments hold
#pragma unroll
  for (int m = 0; m < NT; ++m)
    x4[m] = reinterpret_cast<const uint4*>(p.x + (long long)min(g + 8 * m, T - 1) * K + 32 * t);
  for (int c = warp; c * kChunk < K; c += warps) {
    const uint32_t pa = dq40_pair(s.s0), pb = dq40_pair(s.s1);
    const uint32_t sa = __byte_perm(pa, 0u, 0x1010), ba = __byte_perm(pa, 0u, 0x3232), sa4 = dq40_high(sa);
    const uint32_t sb = __byte_perm(pb, 0u, 0x1010), bb = __byte_perm(pb, 0u, 0x3232), sb4 = dq40_high(sb);
    const uint32_t u0[4] = {s.w0.x, s.w0.y, s.w0.z, s.w0.w}, u1[4] = {s.w1.x, s.w1.y, s.w1.z, s.w1.w};
    const bool in = c * kChunk + 32 * t < K;
    uint4 xv[NT][4];
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) xv[m][q] = in ? x4[m][c * (kChunk / 8) + q] : make_uint4(0u, 0u, 0u, 0u);
    uint4 av[OWN ? 4 : 1][2];
    if (OWN && r)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        av[q][0] = in ? a0[c * (kChunk / 8) + q] : make_uint4(0u, 0u, 0u, 0u);
        av[q][1] = in && r > 8 ? a1[c * (kChunk / 8) + q] : make_uint4(0u, 0u, 0u, 0u);
      }
    fetch(s, c + warps);
    if (OWN && r)
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          mma_bf16(sacc[m], av[q][0].x, av[q][1].x, av[q][0].y, av[q][1].y, xv[m][q].x, xv[m][q].y);
          mma_bf16(sacc[m], av[q][0].z, av[q][1].z, av[q][0].w, av[q][1].w, xv[m][q].z, xv[m][q].w);
        }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t a[2][4];
      dq40_word(u0[q], sa, sa4, ba, a[0][0], a[0][2], a[1][0], a[1][2]);
      dq40_word(u1[q], sb, sb4, bb, a[0][1], a[0][3], a[1][1], a[1][3]);
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        mma_bf16(acc[0][m], a[0][0], a[0][1], a[0][2], a[0][3], xv[m][q].x, xv[m][q].y);
        mma_bf16(acc[kChains - 1][m], a[1][0], a[1][1], a[1][2], a[1][3], xv[m][q].z, xv[m][q].w);
      }
    }
  }
  if (b.after_su) griddep_wait();  // su
  for (int j0 = OWN ? r : 16 * warp; j0 < r; j0 += 16 * warps) {
    if (j0 != 16 * warp) load_adapter(j0, adapter);
    __syncwarp();
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const uint4* su =
          reinterpret_cast<const uint4*>(p.su + (min(g + 8 * m, T - 1) * su_steps(r) + j0 / 16) * kSuWords + 8 * t);
      const uint4 lo = su[0], hi = su[1];
      mma_bf16(acc[0][m], adapter[0], adapter[1], adapter[2], adapter[3], lo.x, hi.x);
      mma_bf16(acc[kChains - 1][m], adapter[0], adapter[1], adapter[2], adapter[3], lo.y, hi.y);
      mma_bf16(acc[0][m], adapter[0], adapter[1], adapter[2], adapter[3], lo.z, hi.z);
    }
  }
  // the warps' sums: [warp][token][row], as large as the block's warps need
  extern __shared__ float red_words[];
  auto red = reinterpret_cast<float(*)[NT * 8][kRedPitch]>(red_words);
#pragma unroll
  for (int m = 0; m < NT; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      red[warp][8 * m + 2 * t + (e & 1)][g + 8 * (e >> 1)] = kChains == 2 ? acc[0][m][e] + acc[kChains - 1][m][e] : acc[0][m][e];
  __shared__ float s_su[OWN ? NT * 8 : 1][16], s_b[OWN ? kTileN : 1][17];
  if constexpr (OWN) {
    const auto su_red = red + warps;
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) su_red[warp][8 * m + 2 * t + (e & 1)][g + 8 * (e >> 1)] = sacc[m][e];
    if (warp == 0)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s_b[g + 8 * (e & 1)][2 * t + 8 * (e >> 1)] = lo_bf16(adapter[e]);
        s_b[g + 8 * (e & 1)][2 * t + 8 * (e >> 1) + 1] = hi_bf16(adapter[e]);
      }
    __syncthreads();
    for (int o = threadIdx.x; o < 16 * T; o += blockDim.x) {
      float v = 0.f;
      for (int w = 0; w < warps; ++w) v += su_red[w][o / 16][o % 16];
      s_su[o / 16][o % 16] = o % 16 < r ? v * p.scale : 0.f;
    }
  }
  __syncthreads();
  for (int o = threadIdx.x; o < kTileN * T; o += blockDim.x) {
    const int tok = o / kTileN, row = o % kTileN, n = n0 + row;
    float v = 0.f;
    for (int w = 0; w < warps; ++w) v += red[w][tok][row];
    v *= 0x1p40f;
    if (OWN && r)
#pragma unroll
      for (int j = 0; j < 16; ++j) v = fmaf(s_su[tok][j], s_b[row][j], v);
    if (n < p.N) p.y[(long long)tok * p.N + n] = __float2bfloat16(v);
  }
}

cudaError_t launch_narrow(DecodeBatch& b, int most, bool own, int num_sms, cudaStream_t st) {
  int tiles = 0, chunks = 1, adapter = 0;  // steps of a block's warps: chunks, and 16 adapter columns
  for (int i = 0; i < b.n; ++i) {
    b.p[i].tile_begin = tiles;
    tiles += (b.p[i].N + kTileN - 1) / kTileN;
    chunks = std::max(chunks, (b.p[i].K + kChunk - 1) / kChunk);
    if (!own) adapter = std::max(adapter, su_steps(b.p[i].r));
  }
  // The steps of a warp (of the adapter's, half), and a quarter of one for each warp that a block's sums come from, times
  // the waves of blocks, of which an SM's registers hold so many (32 warps with 8 tokens, 28 with 16).  (3072 x 5120: 8
  // warps 5.4, 4: 6.7 us; 8192 x 3072: 16: 7.5, 8: 8.5, 4: 12.6; 2048 x 11008: 4: 6.1, 8: 7.6, 2: 8.0; nine tokens,
  // 8192 x 3072: 16, in two waves, 14.8, 13: 11.7; 16 tokens, 64 x 9565, r 128: 1: 11.9, 4: 6.8)
  const int fit = most <= 8 ? 32 : 28;
  int warps = 1;
  double least = 0.0;
  for (int w = 1; w <= kMostThreads / 32 && w <= std::max(chunks, adapter); ++w) {
    const long long at_once = (long long)(fit / w) * num_sms, waves = (tiles + at_once - 1) / at_once;
    const double cost = (double)waves * ((chunks + w - 1) / w + 0.5 * ((adapter + w - 1) / w) + 0.25 * w);
    if (w == 1 || cost < least) {
      warps = w;
      least = cost;
    }
  }
  return with_table(b, [&](const auto& t) {
    using Table = std::decay_t<decltype(t)>;
    const auto kernel = own         ? decode_kernel<1, true, Table>
                        : most <= 8 ? decode_kernel<1, false, Table>
                                    : decode_kernel<2, false, Table>;
    const size_t smem = (size_t)(own ? 2 : 1) * warps * (most <= 8 ? 8 : 16) * kRedPitch * sizeof(float);
    return launch_kernel(kernel, dim3(tiles), dim3(32 * warps), smem, st, 1, t);
  });
}

cudaError_t launch_su(const DecodeBatch& b, int most, cudaStream_t st) {
  return with_table(b, [&](const auto& t) {
    using Table = std::decay_t<decltype(t)>;
    const auto su = most == 1   ? decode_su_kernel<1, Table>
                    : most <= 2 ? decode_su_kernel<2, Table>
                    : most <= 4 ? decode_su_kernel<4, Table>
                    : most <= 8 ? decode_su_kernel<8, Table>
                                : decode_su_kernel<16, Table>;
    return launch_kernel(su, dim3(t.rows), dim3(kSuThreads), 0, st, 1, t);
  });
}

// Which second launch a group of projections takes, by their times as measured (us).  16-row blocks, dealt evenly to the
// SMs, read their bytes at 4.3 TB/s for one token, 3 for eight and 1.8 for sixteen, and are there at once; plan_wide() has
// the wide launch's.  (Blocks and wide, 3072 x 128256, 1 token: 52 and 44, 16: 117 and 45; 4096 x 16384, r 16, 1 token:
// 12.7 and 14.6, 8: 15.9 and 14.7, 16: 22 and 15; 8192 x 8192, r 16, 1 token: 13.0 and 15.0, 8: 16.3 and 15.2, 16: 26 and
// 15.7; two of 2048 x 11008, r 64, 8 tokens: 13.3 and 16.1, 9: 20 and 16.1; 8192 x 3072, r 16, 8 tokens: 9.7 and 10.6, 16:
// 14.0 and 11.7; 3072 x 3072, r 16, 16 tokens: 7.1 and 8.3.)
bool wide_pays(const DecodeBatch& b, int num_sms) {
  const int T = b.p[0].T, K = b.p[0].K;
  long long tiles = 0, blocks = 0;
  int rank = 0;
  for (int i = 0; i < b.n; ++i) {
    tiles += (b.p[i].N + 127) / 128;
    blocks += (b.p[i].N + kTileN - 1) / kTileN;
    rank = std::max(rank, b.p[i].r);
  }
  const double each = (double)((blocks + num_sms - 1) / num_sms);  // of an SM
  const double mb = each * num_sms * kTileN * K * 0.5625e-6;
  const double us = 2.6 + 0.085 * each + mb * (T <= 8 ? 0.22 + 0.0155 * T : 0.27 + 0.018 * T) + 0.02 * rank;
  return plan_wide(tiles, (K + 255) / 256, rank, num_sms).us < us;
}

// Whether the blocks compute su themselves, with all of A read by each of them, against a launch before theirs: a
// launch less costs the host 1.9 us less, which bounds calls this small, and the reading again costs the GPU next to
// nothing up to 4.5 MB of it by one block per SM.  (One token, the GPU alone, then calls in a row; with and without the
// launch before: 256 x 256, r 8, 2.9 and 2.2 us, 5.9 and 4.0; 1024 x 2048, r 16, 4.2 MB, 3.4 and 3.5, 5.9 and 4.0;
// 2048 x 2048, r 8, 4.2 MB, 3.5 and 3.8, 5.9 and 4.1; 3072 x 1024, r 16, 6.3 MB, 4.1 and 5.3, 5.9 and 5.6; 3072 x
// 3072, r 16, 18.9 MB, 4.5 and 7.9, 6.1 and 8.1; 64 x 29768, r 16, 3.8 MB by 1861 blocks, 3.5 and 4.4, with eight tokens
// 3.7 and 6.3.)  More tokens or adapter rows would not fit the registers.
bool own_pays(const DecodeBatch& b, int num_sms) {
  int tiles = 0;
  double again = 0.0;
  for (int i = 0; i < b.n; ++i) {
    const DecodeProj& p = b.p[i];
    if (p.r > 16 || p.T > 8) return false;
    tiles += (p.N + kTileN - 1) / kTileN;
    again += (double)((p.N + kTileN - 1) / kTileN) * p.r * p.K * 2e-6;
  }
  return tiles <= num_sms && again <= 4.5;
}

}  // namespace

size_t decode_su_bytes(int64_t T, int64_t r) {
  return (size_t)T * su_steps((int)r) * kSuWords * 4 + (size_t)kSuTerms * su_blocks((int)r) * kSuBlock;
}

void set_decode_su(DecodeProj& p, void* at) {
  p.su = static_cast<uint32_t*>(at);
  p.su_image = static_cast<uint8_t*>(at) + (size_t)p.T * su_steps(p.r) * kSuWords * 4;
}

cudaError_t launch_decode(DecodeBatch& b, int num_sms, cudaStream_t st) {
  // projections of many rows: one launch for those that read one activation (gate and up); one for all the others
  DecodeBatch rest, same;
  rest.n = rest.rows = same.rows = b.rows = b.after_su = 0;
  rest.status = same.status = b.status;
  rest.limit_ns = same.limit_ns = b.limit_ns;
  int group[kDecodeMaxProjs], most = 1, most_rest = 1;  // the first projection of a wide launch's, or -1
  for (int i = 0; i < b.n; ++i) {
    b.p[i].row_begin = b.rows;
    b.rows += b.p[i].r;
    most = std::max(most, b.p[i].T);
    group[i] = i;
    for (int j = 0; j < i && group[i] == i; ++j)
      if (b.p[j].x == b.p[i].x && b.p[j].T == b.p[i].T && b.p[j].K == b.p[i].K) group[i] = j;
  }
  auto gather = [&](int first) {
    same.n = 0;
    for (int i = first; i < b.n; ++i)
      if (group[i] == first) same.p[same.n++] = b.p[i];
  };
  bool wide[kDecodeMaxProjs], any_wide = false;
  for (int i = 0; i < b.n; ++i) {
    if (group[i] != i) {
      wide[i] = wide[group[i]];
    } else {
      gather(i);
      wide[i] = wide_pays(same, num_sms);
    }
    if (wide[i]) {
      any_wide = true;
    } else {
      rest.p[rest.n++] = b.p[i];
      most_rest = std::max(most_rest, b.p[i].T);
    }
  }
  const bool own = b.rows && !any_wide && own_pays(rest, num_sms);
  rest.after_su = same.after_su = b.rows > 0 && !own;
  if (rest.after_su) {
    const cudaError_t e = launch_su(b, most, st);
    if (e != cudaSuccess) return e;
  }
  for (int i = 0; any_wide && i < b.n; ++i) {
    if (!wide[i] || group[i] != i) continue;
    gather(i);
    const cudaError_t e = launch_decode_wide(same, num_sms, st);
    if (e != cudaSuccess) return e;
  }
  return rest.n ? launch_narrow(rest, most_rest, own, num_sms, st) : cudaSuccess;
}

}  // namespace lora
