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
// Dequantizing takes 9 instructions per 8 codes.  A bf16 whose exponent field is 0 or 1 is its low 8 bits as an
// integer, times 2^-133: the codes in bits 0..3 and 16..19 of a word are a pair of bf16 q * 2^-133 as they lie, those
// in bits 4..7 and 20..23 a pair 16 q * 2^-133.  One FMA with s * 2^93 (or s * 2^89) and b * 2^-40 then gives
// 2^-40 (s q + b), rounded to bf16 once like the training kernels' weight, and the sums are scaled back by 2^40.
// (Valid for |s| < 2^35; a weight below 2^-86 loses bits.)
//
// su enters the same MMAs as three bf16 terms, which hold all 24 bits of its fp32 value.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace lora {
namespace {

constexpr int kTileN = 16;       // output rows of a tile: M of the MMA
constexpr int kChunk = 128;      // columns of a warp's step: two 64-wide groups, 32 columns a lane
constexpr int kWarps = 16, kThreads = 32 * kWarps;  // one CTA per SM
constexpr int kAhead = 4;        // steps of a warp on their way
constexpr int kRedPitch = 20;    // floats: the partial sums' stores meet no bank twice
constexpr size_t kMostSmem = 227 * 1024;
constexpr int kXPad = 64;        // bytes behind each token's row: tokens alternate between the banks' halves

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) { return fma_bf16x2(a, b, 0x80008000u); }

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// su as the MMAs' B operand reads it, for 16 adapter columns at a time: [T][su_steps(r)][t][8 words], where lane t's
// words 0..2 hold columns 2 t and 2 t + 1 in three terms, and words 4..6 columns 2 t + 8 and 2 t + 9.  Times 2^-40 like
// the weights, zeros behind column r.
constexpr int kSuTerms = 3, kSuWords = 32;
__host__ __device__ constexpr int su_steps(int r) { return (r + 15) / 16; }
__device__ __forceinline__ int su_at(int r, int tok, int col, int term) {  // in 16-bit units
  const int c = col & 15;
  return 2 * ((tok * su_steps(r) + col / 16) * kSuWords + (c & 7) / 2 * 8 + c / 8 * 4 + term) + (c & 1);
}

// One block per (projection, adapter row j): su[t, j] = scale * x_t . A_j for up to TT tokens.
constexpr int kSuThreads = 256;
template <int TT>
__global__ void __launch_bounds__(kSuThreads) decode_su_kernel(const __grid_constant__ DecodeBatch b) {
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
    __nv_bfloat16* su = reinterpret_cast<__nv_bfloat16*>(p.su);
#pragma unroll
    for (int e = 0; e < kSuTerms; ++e) {
      const __nv_bfloat16 term = __float2bfloat16(v);
      su[su_at(p.r, threadIdx.x, j, e)] = term;
      v = isfinite(v) ? v - __bfloat162float(term) : 0.f;
    }
    if (j == p.r - 1)
      for (int col = p.r; col < 16 * su_steps(p.r); ++col)
        for (int e = 0; e < kSuTerms; ++e) su[su_at(p.r, threadIdx.x, col, e)] = __float2bfloat16(0.f);
  }
}

// What one warp reads per step: 32 codes of row g and of row g + 8 for each lane (g, t), with their (s, b).
struct Step {
  uint4 w0, w1;
  uint32_t s0, s1;
};

// Loads a step where `ok`.  Elsewhere s = b = 0 make the weights zero whatever the codes' registers hold.
__device__ __forceinline__ void load_step(Step& s, bool ok, const uint8_t* codes, int codes1, const uint32_t* params,
                                          int params1) {
  s.s0 = s.s1 = 0u;
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %14, 0;\n\t"
      "@p ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%10];\n\t"
      "@p ld.global.nc.L1::no_allocate.v4.u32 {%4, %5, %6, %7}, [%11];\n\t"
      "@p ld.global.nc.u32 %8, [%12];\n\t"
      "@p ld.global.nc.u32 %9, [%13];\n\t}"
      : "=r"(s.w0.x), "=r"(s.w0.y), "=r"(s.w0.z), "=r"(s.w0.w), "=r"(s.w1.x), "=r"(s.w1.y), "=r"(s.w1.z),
        "=r"(s.w1.w), "+r"(s.s0), "+r"(s.s1)
      : "l"(codes), "l"(codes + codes1), "l"(params), "l"(params + params1), "r"((uint32_t)ok));
}

__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}

// `split` warps share a tile of 16 rows: warp i of them has every split-th chunk of the columns from i on, and every
// split-th 16 of the adapter's, and the warps' sums meet in shared memory (split 1: a warp stores its own).  Tiles go
// round the SMs first.  A lane's word of 8 codes makes the fragments of two MMAs, whose k index is then a permutation
// of the columns; the activation's fragments share it: 16 consecutive bytes of token g.  kAhead steps per warp are on
// their way while one is computed, also across tiles.  The activation stays in shared memory (XS; where its T rows
// do not fit, its fragments come through L1).
template <int NT, bool XS>  // NT: tokens / 8
__global__ void __launch_bounds__(kThreads) decode_kernel(const __grid_constant__ DecodeBatch b, int split) {
  extern __shared__ __align__(16) uint8_t smem[];
  float* red = reinterpret_cast<float*>(smem);  // split > 1: [kWarps][NT * 8][kRedPitch]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int group = warp / split, wg = warp % split;
  const int slot = group * (int)gridDim.x + (int)blockIdx.x, slots = kWarps / split * (int)gridDim.x;
  const int T = b.p[0].T, K = b.p[0].K;
  const __nv_bfloat16* x = b.p[0].x;
  if (!b.after_su) griddep_wait();  // otherwise the launch before is this call's, and began after its inputs were there
  griddep_launch_dependents();
  bool waited = !b.after_su;

  // the loads' cursor, ahead of the computation's
  int l_tile = slot, l_proj = 0, l_c = wg;
  const uint8_t* codes = nullptr;
  const uint32_t* params = nullptr;
  int codes1 = 0, params1 = 0;  // from row g to row g + 8 (rows past the last: the last)
  auto l_open = [&]() {
    l_c = wg;
    if (l_tile >= b.tiles) return;
    while (l_proj + 1 < b.n && l_tile >= b.p[l_proj + 1].tile_begin) ++l_proj;
    const DecodeProj& p = b.p[l_proj];
    const int n0 = (l_tile - p.tile_begin) * kTileN, r0 = min(n0 + g, p.N - 1), r1 = min(n0 + g + 8, p.N - 1);
    codes = p.codes + (long long)r0 * (K / 2) + wg * (kChunk / 2) + 16 * t;
    params = reinterpret_cast<const uint32_t*>(p.params) + (long long)r0 * (K / 64) + wg * (kChunk / 64) + t / 2;
    codes1 = (r1 - r0) * (K / 2);
    params1 = (r1 - r0) * (K / 64);
  };
  auto fetch = [&](Step& s) {
    // K is a multiple of 64: the last chunk may be half a one
    load_step(s, l_tile < b.tiles && l_c * kChunk + 32 * t < K, codes, codes1, params, params1);
    l_c += split;
    codes += split * (kChunk / 2);
    params += split * (kChunk / 64);
    if (l_c * kChunk >= K) {
      l_tile += slots;
      l_open();
    }
  };
  l_open();
  Step steps[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(steps[i]);

  // columns past T are dropped: whatever token their fragments hold
  uint32_t xs[NT];  // shared address of the lane's fragments of the first chunk
  if (XS) {
    uint8_t* held = smem + (split > 1 ? kWarps * NT * 8 * kRedPitch * 4 : 0);
    const int units = (K + kChunk - 1) / kChunk * (kChunk / 8), have = K / 8;  // 16 bytes each
    const int pitch = units * 16 + kXPad;
    for (int tok = 0; tok < T; ++tok)
      for (int v = threadIdx.x; v < units; v += kThreads) {
        const uint4 d =
            v < have ? reinterpret_cast<const uint4*>(x + (long long)tok * K)[v] : make_uint4(0u, 0u, 0u, 0u);
        // unit 4 t + q of a chunk lies at 4 q + t: the lanes of a fragment's load read 64 consecutive bytes a token
        *reinterpret_cast<uint4*>(held + tok * pitch + ((v & ~15) + 4 * (v & 3) + (v >> 2 & 3)) * 16) = d;
      }
#pragma unroll
    for (int m = 0; m < NT; ++m) xs[m] = smem_u32(held) + min(g + 8 * m, T - 1) * pitch + 16 * t;
    __syncthreads();
  }

  float acc[NT][4];
  int c = wg;
  // One step: its products, and the next load into its place; true behind the tile's last.
  auto step = [&](Step& s) {
    const uint32_t pa = mul_bf16x2(s.s0, 0x2B806E00u), pb = mul_bf16x2(s.s1, 0x2B806E00u);  // 2^93, 2^-40
    const uint32_t sa = __byte_perm(pa, 0u, 0x1010), ba = __byte_perm(pa, 0u, 0x3232);
    const uint32_t sb = __byte_perm(pb, 0u, 0x1010), bb = __byte_perm(pb, 0u, 0x3232);
    const uint32_t sa4 = mul_bf16x2(sa, 0x3D803D80u), sb4 = mul_bf16x2(sb, 0x3D803D80u);  // 1/16
    const uint32_t u0[4] = {s.w0.x, s.w0.y, s.w0.z, s.w0.w};
    const uint32_t u1[4] = {s.w1.x, s.w1.y, s.w1.z, s.w1.w};
    fetch(s);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint4 xv[NT];
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        if (XS)
          xv[m] = load_shared(xs[m] + c * (kChunk * 2) + 64 * q);
        else
          xv[m] = c * kChunk + 32 * t < K
                      ? __ldg(reinterpret_cast<const uint4*>(x + (long long)min(g + 8 * m, T - 1) * K + c * kChunk +
                                                             32 * t + 8 * q))
                      : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t v0 = h ? u0[q] >> 8 : u0[q], v1 = h ? u1[q] >> 8 : u1[q];
        const uint32_t a0 = fma_bf16x2(v0 & 0x000F000Fu, sa, ba), a1 = fma_bf16x2(v1 & 0x000F000Fu, sb, bb);
        const uint32_t a2 = fma_bf16x2(v0 & 0x00F000F0u, sa4, ba), a3 = fma_bf16x2(v1 & 0x00F000F0u, sb4, bb);
#pragma unroll
        for (int m = 0; m < NT; ++m)
          mma_bf16(acc[m], a0, a1, a2, a3, h ? xv[m].z : xv[m].x, h ? xv[m].w : xv[m].y);
      }
    }
    c += split;
    return c * kChunk >= K;
  };
  auto sync_group = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * split) : "memory"); };

  int proj = 0, pos = 0;
  for (int tile = slot; tile < b.tiles; tile += slots) {
    while (proj + 1 < b.n && tile >= b.p[proj + 1].tile_begin) ++proj;
    const DecodeProj& p = b.p[proj];
    const int n0 = (tile - p.tile_begin) * kTileN, r = p.r;
    // the adapter's A operand of 16 columns: rows g and g + 8 of B, columns 2 t (+ 1) and 2 t + 8 (+ 9)
    auto load_adapter = [&](int j0, uint32_t (&a)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + g + 8 * (i & 1), j = j0 + 2 * t + 8 * (i >> 1);
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p.B) + (long long)n * r + j;
        a[i] = 0u;
        if (n < p.N && j < r) {
          if (r % 2 == 0)
            a[i] = __ldg(reinterpret_cast<const uint32_t*>(q));
          else
            a[i] = __ldg(q) | (j + 1 < r ? (uint32_t)__ldg(q + 1) << 16 : 0u);
        }
      }
    };
    uint32_t adapter[4];
    load_adapter(16 * wg, adapter);
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[m][e] = 0.f;
    c = wg;
    for (bool done = false; !done;) {
      switch (pos) {
        case 0:
          pos = 1;
          if ((done = step(steps[0]))) break;
          [[fallthrough]];
        case 1:
          pos = 2;
          if ((done = step(steps[1]))) break;
          [[fallthrough]];
        case 2:
          pos = 3;
          if ((done = step(steps[2]))) break;
          [[fallthrough]];
        default:
          pos = 0;
          done = step(steps[3]);
      }
    }
    for (int j0 = 16 * wg; j0 < r; j0 += 16 * split) {
      if (!waited) {
        griddep_wait();  // su
        waited = true;
      }
      if (j0 != 16 * wg) load_adapter(j0, adapter);
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        const uint4* su =
            reinterpret_cast<const uint4*>(p.su + (min(g + 8 * m, T - 1) * su_steps(r) + j0 / 16) * kSuWords + 8 * t);
        const uint4 lo = su[0], hi = su[1];
        mma_bf16(acc[m], adapter[0], adapter[1], adapter[2], adapter[3], lo.x, hi.x);
        mma_bf16(acc[m], adapter[0], adapter[1], adapter[2], adapter[3], lo.y, hi.y);
        mma_bf16(acc[m], adapter[0], adapter[1], adapter[2], adapter[3], lo.z, hi.z);
      }
    }
    if (split == 1) {
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = 8 * m + 2 * t + (e & 1), n = n0 + g + 8 * (e >> 1);
          if (tok < T && n < p.N) p.y[(long long)tok * p.N + n] = __float2bfloat16(acc[m][e] * 0x1p40f);
        }
      continue;
    }
    sync_group();  // the sums of the tile before are read
    float* mine = red + warp * (NT * 8 * kRedPitch);
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[(8 * m + 2 * t + (e & 1)) * kRedPitch + g + 8 * (e >> 1)] = acc[m][e];
    sync_group();
    const float* sums = red + group * split * (NT * 8 * kRedPitch);
    for (int o = wg * 32 + lane; o < kTileN * T; o += 32 * split) {
      const int tok = o / kTileN, row = o % kTileN, n = n0 + row;
      float v = 0.f;
#pragma unroll 4
      for (int w = 0; w < split; ++w) v += sums[(w * NT * 8 + tok) * kRedPitch + row];
      if (n < p.N) p.y[(long long)tok * p.N + n] = __float2bfloat16(v * 0x1p40f);
    }
  }
  if (!waited) griddep_wait();  // no grid ends before the ones it follows
}

// Warps per tile.  More of them finish a tile sooner, fewer share less: the cost of a choice is the rounds of the
// SMs' slots, times the chunks of a warp and what its end takes, in chunks.
int choose_split(int tiles, int chunks, int num_sms) {
  int best = 1;
  double least = 0.0;
  for (int split = 1; split <= kWarps && split <= chunks; split *= 2) {
    const int slots = num_sms * (kWarps / split);
    const double cost = (double)((tiles + slots - 1) / slots) * ((chunks + split - 1) / split + (split == 1 ? 0.5 : 1.5));
    if (split == 1 || cost < least) {
      best = split;
      least = cost;
    }
  }
  return best;
}

template <int NT, bool XS>
cudaError_t launch_main(const DecodeBatch& b, int split, size_t smem, int num_sms, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = set_smem_once(decode_kernel<NT, XS>, kMostSmem, done);
  if (e != cudaSuccess) return e;
  return launch_kernel(decode_kernel<NT, XS>, dim3(std::min(b.tiles, num_sms)), dim3(kThreads), smem, st, 1, b, split);
}

template <int NT>
cudaError_t launch_main(const DecodeBatch& b, int num_sms, cudaStream_t st) {
  const int chunks = (b.p[0].K + kChunk - 1) / kChunk, split = choose_split(b.tiles, chunks, num_sms);
  const size_t red = split > 1 ? (size_t)kWarps * NT * 8 * kRedPitch * 4 : 0;
  const size_t held = (size_t)b.p[0].T * (chunks * (kChunk * 2) + kXPad);
  return red + held <= kMostSmem ? launch_main<NT, true>(b, split, red + held, num_sms, st)
                                 : launch_main<NT, false>(b, split, red, num_sms, st);
}

cudaError_t launch_su(const DecodeBatch& b, int most, cudaStream_t st) {
  const auto su = most == 1   ? decode_su_kernel<1>
                  : most <= 2 ? decode_su_kernel<2>
                  : most <= 4 ? decode_su_kernel<4>
                  : most <= 8 ? decode_su_kernel<8>
                              : decode_su_kernel<16>;
  return launch_kernel(su, dim3(b.rows), dim3(kSuThreads), 0, st, 1, b);
}

}  // namespace

size_t decode_su_bytes(int64_t T, int64_t r) { return (size_t)T * su_steps((int)r) * kSuWords * 4; }

cudaError_t launch_decode(DecodeBatch& b, int num_sms, cudaStream_t st) {
  b.rows = 0;
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
  // one launch for the projections that read one activation: q, k and v; gate and up
  bool taken[kDecodeMaxProjs] = {};
  for (int i = 0; i < b.n; ++i) {
    if (taken[i]) continue;
    DecodeBatch same;
    same.n = same.tiles = 0;
    same.after_su = b.rows > 0;
    for (int j = i; j < b.n; ++j) {
      if (taken[j] || b.p[j].x != b.p[i].x || b.p[j].T != b.p[i].T || b.p[j].K != b.p[i].K) continue;
      taken[j] = true;
      DecodeProj& p = same.p[same.n++];
      p = b.p[j];
      p.tile_begin = same.tiles;
      same.tiles += (p.N + kTileN - 1) / kTileN;
    }
    const cudaError_t e = b.p[i].T <= 8 ? launch_main<1>(same, num_sms, st) : launch_main<2>(same, num_sms, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace lora
