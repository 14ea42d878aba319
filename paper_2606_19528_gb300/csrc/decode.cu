// Forward of adapted projections with 4-bit weights for 1 to 16 tokens:
//   decode_su_kernel  su = scale * x A^T, one block per adapter row
//   decode_kernel     y  = x W^T + su B^T, W[n, k] = bf16(s q + b) from its 4-bit codes
//
// With so few tokens every weight is used once or a handful of times, so the call is bound by reading 9/16 byte per
// weight, and next by the instructions that dequantize it.  The products go through mma.sync m16n8k16, whose 8
// columns are the tokens: an accumulation on the FMA units would take two conversions and 2 T FMAs per pair of
// weights more, and the tcgen05 path wants its operands in shared memory, where the round trip of the dequantized
// weights alone costs more than the products of 16 tokens.
//
// Dequantizing takes 9 instructions per 8 codes (dq40_word); the sums are scaled back by 2^40.
//
// su enters the same MMAs as three bf16 terms, which hold all 24 bits of its fp32 value.
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
// two to four steps ahead takes the registers of as many warps and is slower.  A lane's word of 8 codes makes the fragments of two MMAs, whose k index is
// then a permutation of the columns; the activation's fragments share it: 16 consecutive bytes of token g, which come
// through L1.
template <int NT, typename Table>  // tokens / 8
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
          a[e] = __ldg(reinterpret_cast<const uint32_t*>(q));
        else
          a[e] = __ldg(q) | (j + 1 < r ? (uint32_t)__ldg(q + 1) << 16 : 0u);
      }
    }
  };
  uint32_t adapter[4];
  load_adapter(16 * warp, adapter);

  float acc[kChains][NT][4] = {};
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
      for (int q = 0; q < 4; ++q) xv[m][q] = in ? __ldg(x4[m] + c * (kChunk / 8) + q) : make_uint4(0u, 0u, 0u, 0u);
    fetch(s, c + warps);
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
  for (int j0 = 16 * warp; j0 < r; j0 += 16 * warps) {
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
  __shared__ float red[kMostThreads / 32][NT * 8][kRedPitch];
#pragma unroll
  for (int m = 0; m < NT; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      red[warp][8 * m + 2 * t + (e & 1)][g + 8 * (e >> 1)] = kChains == 2 ? acc[0][m][e] + acc[kChains - 1][m][e] : acc[0][m][e];
  __syncthreads();
  for (int o = threadIdx.x; o < kTileN * T; o += blockDim.x) {
    const int tok = o / kTileN, row = o % kTileN, n = n0 + row;
    float v = 0.f;
    for (int w = 0; w < warps; ++w) v += red[w][tok][row];
    if (n < p.N) p.y[(long long)tok * p.N + n] = __float2bfloat16(v * 0x1p40f);
  }
}

cudaError_t launch_narrow(DecodeBatch& b, int most, int num_sms, cudaStream_t st) {
  int tiles = 0, chunks = 1;
  for (int i = 0; i < b.n; ++i) {
    b.p[i].tile_begin = tiles;
    tiles += (b.p[i].N + kTileN - 1) / kTileN;
    chunks = std::max(chunks, (b.p[i].K + kChunk - 1) / kChunk);
  }
  // The steps of a warp, and about a quarter of one for each warp that a block's sums come from, times the waves of
  // blocks (about 30 warps fit an SM).  (3072 x 5120: 8 warps 5.4, 4: 6.7 us; 8192 x 3072: 16: 7.5, 8: 8.5, 4: 12.6 us;
  // 2048 x 11008: 4: 6.1, 8: 7.6, 2: 8.0 us)
  int warps = 1;
  double least = 0.0;
  for (int w = 1; w <= kMostThreads / 32 && w <= chunks; ++w) {
    const long long waves = ((long long)tiles * w + 30 * num_sms - 1) / (30 * num_sms);
    const double cost = (double)waves * ((chunks + w - 1) / w + 0.25 * w);
    if (w == 1 || cost < least) {
      warps = w;
      least = cost;
    }
  }
  return with_table(b, [&](const auto& t) {
    using Table = std::decay_t<decltype(t)>;
    return launch_kernel(most <= 8 ? decode_kernel<1, Table> : decode_kernel<2, Table>, dim3(tiles), dim3(32 * warps), 0,
                         st, 1, t);
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

// Which second launch a group of projections takes, by their times as measured (us): 16-row blocks read their bytes at
// 4.3 TB/s for one token, 3 for eight and 1.8 for sixteen, and are there at once; the wide launch takes 0.475 for a
// panel of 128 rows whatever the tokens, and starts late.  (3072 x 128256, 1 and 16 tokens: blocks 52 and 117, wide 44
// and 45; 3072 x 16384: 9.0 and 19, 10.9 and 11.3; 8192 x 3072: 8.4 and 13.7, 19 and 20; 4096 x 16384, 8 tokens: 15.5,
// 13.0.)
bool wide_pays(const DecodeBatch& b, int num_sms) {
  const int T = b.p[0].T, K = b.p[0].K;
  double mb = 0.0;
  long long tiles = 0;
  int adapters = 0;
  for (int i = 0; i < b.n; ++i) {
    mb += (double)b.p[i].N * K * (0.5625e-6);
    tiles += (b.p[i].N + 127) / 128;
    adapters |= b.p[i].r > 0;
  }
  const double blocks = 2.6 + mb * (T <= 8 ? 0.22 + 0.0155 * T : 0.27 + 0.018 * T);
  const double wide = 4.6 + (double)((tiles + num_sms - 1) / num_sms) * ((K + 255) / 256 + adapters) * 0.475;
  return wide < blocks;
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
  b.rows = b.after_su = 0;
  int most = 1;
  for (int i = 0; i < b.n; ++i) {
    b.p[i].row_begin = b.rows;
    b.rows += b.p[i].r;
    most = std::max(most, b.p[i].T);
  }
  if (b.rows) {
    const cudaError_t e = launch_su(b, most, st);
    if (e != cudaSuccess) return e;
  }
  // projections of many rows: one launch for those that read one activation (gate and up); one for all the others
  DecodeBatch rest, same;
  rest.n = rest.rows = same.rows = 0;
  rest.after_su = same.after_su = b.rows > 0;
  rest.status = same.status = b.status;
  rest.limit_ns = same.limit_ns = b.limit_ns;
  bool taken[kDecodeMaxProjs] = {};
  most = 1;
  for (int i = 0; i < b.n; ++i) {
    if (taken[i]) continue;
    same.n = 0;
    for (int j = i; j < b.n; ++j) {
      if (taken[j] || b.p[j].x != b.p[i].x || b.p[j].T != b.p[i].T || b.p[j].K != b.p[i].K) continue;
      taken[j] = true;
      same.p[same.n++] = b.p[j];
    }
    if (wide_pays(same, num_sms)) {
      const cudaError_t e = launch_decode_wide(same, num_sms, st);
      if (e != cudaSuccess) return e;
    } else {
      for (int j = 0; j < same.n; ++j) rest.p[rest.n++] = same.p[j];
      most = std::max(most, b.p[i].T);
    }
  }
  return rest.n ? launch_narrow(rest, most, num_sms, st) : cudaSuccess;
}

}  // namespace lora
