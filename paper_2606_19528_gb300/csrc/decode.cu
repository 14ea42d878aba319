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
constexpr int kPanel = 256;      // columns of a warp's step: a 64-wide group to each of the four lanes of a row
constexpr int kWarps = 16, kThreads = 32 * kWarps;  // one CTA per SM
constexpr int kMaxStages = 8;
constexpr int kCtlBytes = 128;
constexpr long long kAbortDrainNs = 2000000;
constexpr int kRedPitch = 20;    // floats: the partial sums' stores meet no bank twice
constexpr int kMostSmem = 227 * 1024;
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

// How a launch cuts its work.  A tile is MT * 16 rows; `split` warps share a group's tiles, each taking every split-th
// panel of 256 columns, with `stages` panels of codes on their way or in use.
struct Cut {
  int split, groups, stages, tiles;
  int red_bytes, held_bytes;  // of the warps' sums, the activation
};

// Each warp keeps a ring of its own filled by tiled copies (a tile's rows and a panel's columns, 128-byte swizzle, zeros
// outside the matrix), so that no warp waits for another but at the end of a tile that several share.  Tiles go round
// the SMs first.
// A lane has the 64 columns of one (s, b) pair of rows g and g + 8: a word of 8 codes makes the fragments of two MMAs,
// whose k index is then a permutation of the columns; the activation's fragments share it, 16 consecutive bytes of
// token g.  The warps of a group also share out the adapter's columns by 16, and their sums meet in shared memory
// (split 1: a warp stores its own).  The activation stays in shared memory (XS; where its T rows do not fit, its
// fragments come through L1).
template <int NT, int MT, bool XS>  // NT: tokens / 8; MT: sixteens of rows per tile, which share the activation's fragments
__global__ void __launch_bounds__(kThreads) decode_kernel(const __grid_constant__ DecodeBatch b,
                                                          const __grid_constant__ Cut cut) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr int kChains = NT * MT == 1 ? 2 : 1;  // of dependent MMAs: two at least
  constexpr int kRows = MT * kTileN;
  constexpr uint32_t kStageBytes = kRows * (kPanel / 2);
  const int split = cut.split, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int active = cut.groups * split;
  const int T = b.p[0].T, K = b.p[0].K, panels = (K + kPanel - 1) / kPanel, pairs = K / 64;
  uint8_t* red_at = smem + active * cut.stages * kStageBytes;
  uint8_t* held = red_at + cut.red_bytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(held + cut.held_bytes);
  int* abort_word = reinterpret_cast<int*>(bars + active * cut.stages);
  if (threadIdx.x == 0) {
    for (int i = 0; i < active * cut.stages; ++i) mbar_init(smem_u32(bars + i), 1);
    *abort_word = 0;
    fence_mbar_init();
  }
  __syncthreads();
  if (!b.after_su) griddep_wait();  // otherwise the launch before is this call's, and began after its inputs were there
  griddep_launch_dependents();
  if (warp >= active) return;

  const int group = warp / split, wg = warp % split;
  const int slots = cut.groups * (int)gridDim.x, slot = group * (int)gridDim.x + (int)blockIdx.x;
  const uint32_t ring_at = warp * cut.stages * kStageBytes;  // from smem
  const uint32_t ring = smem_u32(smem) + ring_at, bar = smem_u32(bars + warp * cut.stages);
  const WaitCtl wait{b.status, b.limit_ns};
  volatile int* abort = abort_word;

  // copies: the cursor of the next one to issue (lane 0)
  int l_tile = slot, l_proj = 0, l_c = wg, issued = 0;
  auto issue = [&](int s) {
    if (l_tile >= cut.tiles) return;
    while (l_proj + 1 < b.n && l_tile >= b.p[l_proj + 1].tile_begin) ++l_proj;
    mbar_arrive_expect_tx(bar + 8 * s, kStageBytes);
    tma_load_2d(ring + s * kStageBytes, &b.codes[l_proj], bar + 8 * s, l_c * (kPanel / 2),
                (l_tile - b.p[l_proj].tile_begin) * kRows);
    ++issued;
    l_c += split;
    if (l_c >= panels) {
      l_c = wg;
      l_tile += slots;
    }
  };
  if (lane == 0)
    for (int s = 0; s < cut.stages; ++s) issue(s);

  // (s, b) pairs, loaded a step ahead: the cursor of the next step's
  int q_tile = slot, q_proj = 0, q_c = wg;
  const uint32_t* q_at = nullptr;  // of row g, 8 rows being `pairs` * 8 words
  int q_rows = 0;                  // rows of the matrix from the tile's first on
  auto q_open = [&]() {
    if (q_tile >= cut.tiles) {
      q_rows = 0;
      return;
    }
    while (q_proj + 1 < b.n && q_tile >= b.p[q_proj + 1].tile_begin) ++q_proj;
    const DecodeProj& p = b.p[q_proj];
    const int n0 = (q_tile - p.tile_begin) * kRows;
    q_rows = p.N - n0;
    q_at = reinterpret_cast<const uint32_t*>(p.params) + (long long)(n0 + g) * pairs + t;
  };
  uint32_t next_pair[2 * MT];
  auto fetch_pairs = [&]() {
    const bool in = 4 * q_c + t < pairs;  // the last panel may be a part of one
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i)
      next_pair[i] = in && g + 8 * i < q_rows ? __ldg(q_at + 4 * q_c + i * 8 * pairs) : 0u;
    q_c += split;
    if (q_c >= panels) {
      q_c = wg;
      q_tile += slots;
      q_open();
    }
  };
  q_open();
  fetch_pairs();

  const __nv_bfloat16* x = b.p[0].x;
  // columns past T are dropped: whatever token their fragments hold
  uint32_t xs[NT];  // where the lane's fragments of the first panel lie, from smem
  if (XS) {
    const int units = panels * (kPanel / 8), have = K / 8, x_pitch = units * 16 + kXPad;  // units of 16 bytes of a token
    for (int tok = 0; tok < T; ++tok)
      for (int v = threadIdx.x; v < units; v += 32 * active) {
        const uint4 d =
            v < have ? reinterpret_cast<const uint4*>(x + (long long)tok * K)[v] : make_uint4(0u, 0u, 0u, 0u);
        // unit 8 t + q of a panel lies at 4 q + t: the lanes of a fragment's load read 64 consecutive bytes a token
        *reinterpret_cast<uint4*>(held + tok * x_pitch + ((v & ~31) + 4 * (v & 7) + (v >> 3 & 3)) * 16) = d;
      }
#pragma unroll
    for (int m = 0; m < NT; ++m) xs[m] = (uint32_t)(held - smem) + min(g + 8 * m, T - 1) * x_pitch + 16 * t;
    __syncwarp();
    asm volatile("bar.sync 15, %0;" ::"r"(32 * active) : "memory");
  }
  // 16-byte units 2 t and 2 t + 1 of a row's 128 bytes, swizzled by the row (its last three bits are g's)
  const uint32_t even = ring_at + g * (kPanel / 2) + ((2 * t) ^ g) * 16;
  const uint32_t odd = ring_at + g * (kPanel / 2) + ((2 * t + 1) ^ g) * 16;
  bool waited = !b.after_su, alive = true;
  int s = 0, proj = 0;
  uint32_t phase = 0;
  for (int tile = slot; tile < cut.tiles; tile += slots) {
    while (proj + 1 < b.n && tile >= b.p[proj + 1].tile_begin) ++proj;
    const DecodeProj& p = b.p[proj];
    const int n0 = (tile - p.tile_begin) * kRows, r = p.r;
    // the adapter's A operand of 16 columns: rows g and g + 8 of B, columns 2 t (+ 1) and 2 t + 8 (+ 9)
    auto load_adapter = [&](int mt, int j0, uint32_t (&a)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + mt * kTileN + g + 8 * (i & 1), j = j0 + 2 * t + 8 * (i >> 1);
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
    uint32_t adapter[MT][4];  // its first columns, on their way meanwhile
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) load_adapter(mt, 16 * wg, adapter[mt]);
    float acc[kChains][MT][NT][4] = {};
    for (int c = wg; c < panels; c += split) {
      uint32_t sc[MT][2], sc4[MT][2], of[MT][2];
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) {  // eights of rows
        const uint32_t sb = mul_bf16x2(next_pair[i], 0x2B806E00u);  // 2^93, 2^-40
        sc[i / 2][i % 2] = __byte_perm(sb, 0u, 0x1010);
        of[i / 2][i % 2] = __byte_perm(sb, 0u, 0x3232);
        sc4[i / 2][i % 2] = mul_bf16x2(sc[i / 2][i % 2], 0x3D803D80u);  // 1/16
      }
      fetch_pairs();
      if (alive) alive = mbar_wait(bar + 8 * s, phase, wait, abort);
      __syncwarp();  // the MMAs need the warp whole
      const uint32_t at = s * kStageBytes, xc = c * (kPanel * 2);
#pragma unroll
      for (int half = 0; half < 2; ++half) {  // a lane's first 32 columns and its last
        uint4 w[MT][2];
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i)
          w[i / 2][i % 2] = *reinterpret_cast<const uint4*>(smem + at + (half ? odd : even) + i * 8 * (kPanel / 2));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint4 xv[NT];
#pragma unroll
          for (int m = 0; m < NT; ++m) {
            if (XS)
              xv[m] = *reinterpret_cast<const uint4*>(smem + xs[m] + xc + 256 * half + 64 * q);
            else
              xv[m] = 4 * c + t < pairs ? __ldg(reinterpret_cast<const uint4*>(
                                              x + (long long)min(g + 8 * m, T - 1) * K + c * kPanel + 64 * t + 32 * half +
                                              8 * q))
                                        : make_uint4(0u, 0u, 0u, 0u);
          }
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const uint4 w0 = w[mt][0], w1 = w[mt][1];
            const uint32_t u0 = q == 0 ? w0.x : q == 1 ? w0.y : q == 2 ? w0.z : w0.w;
            const uint32_t u1 = q == 0 ? w1.x : q == 1 ? w1.y : q == 2 ? w1.z : w1.w;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t v0 = h ? u0 >> 8 : u0, v1 = h ? u1 >> 8 : u1;
              const uint32_t a0 = fma_bf16x2(v0 & 0x000F000Fu, sc[mt][0], of[mt][0]);
              const uint32_t a1 = fma_bf16x2(v1 & 0x000F000Fu, sc[mt][1], of[mt][1]);
              const uint32_t a2 = fma_bf16x2(v0 & 0x00F000F0u, sc4[mt][0], of[mt][0]);
              const uint32_t a3 = fma_bf16x2(v1 & 0x00F000F0u, sc4[mt][1], of[mt][1]);
#pragma unroll
              for (int m = 0; m < NT; ++m)
                mma_bf16(acc[h % kChains][mt][m], a0, a1, a2, a3, h ? xv[m].z : xv[m].x, h ? xv[m].w : xv[m].y);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0 && alive) issue(s);
      if (++s == cut.stages) {
        s = 0;
        phase ^= 1u;
      }
    }
    if (kChains == 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[0][0][0][e] += acc[kChains - 1][0][0][e];
    }
    for (int j0 = 16 * wg; j0 < r; j0 += 16 * split) {
      if (!waited) {
        griddep_wait();  // su
        waited = true;
      }
      uint4 lo[NT], hi[NT];
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        const uint4* su =
            reinterpret_cast<const uint4*>(p.su + (min(g + 8 * m, T - 1) * su_steps(r) + j0 / 16) * kSuWords + 8 * t);
        lo[m] = su[0];
        hi[m] = su[1];
      }
      __syncwarp();
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (j0 != 16 * wg) load_adapter(mt, j0, adapter[mt]);
        __syncwarp();
        const uint32_t(&a)[4] = adapter[mt];
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          mma_bf16(acc[0][mt][m], a[0], a[1], a[2], a[3], lo[m].x, hi[m].x);
          mma_bf16(acc[0][mt][m], a[0], a[1], a[2], a[3], lo[m].y, hi[m].y);
          mma_bf16(acc[0][mt][m], a[0], a[1], a[2], a[3], lo[m].z, hi[m].z);
        }
      }
    }
    auto sync_group = [&]() {
      __syncwarp();  // a warp in parts would count as several
      asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * split) : "memory");
    };
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (split == 1) {
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = 8 * m + 2 * t + (e & 1), n = n0 + mt * kTileN + g + 8 * (e >> 1);
            if (tok < T && n < p.N) p.y[(long long)tok * p.N + n] = __float2bfloat16(acc[0][mt][m][e] * 0x1p40f);
          }
        continue;
      }
      float* red = reinterpret_cast<float*>(red_at);  // [active][NT * 8][kRedPitch]
      float* mine = red + warp * (NT * 8 * kRedPitch);
      sync_group();  // the sums of the tile before are read
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[(8 * m + 2 * t + (e & 1)) * kRedPitch + g + 8 * (e >> 1)] = acc[0][mt][m][e];
      sync_group();
      const float* sums = red + group * split * (NT * 8 * kRedPitch);
      for (int o = wg * 32 + lane; o < kTileN * T; o += 32 * split) {
        const int tok = o / kTileN, row = o % kTileN, n = n0 + mt * kTileN + row;
        float v = 0.f;
#pragma unroll 4
        for (int w = 0; w < split; ++w) v += sums[(w * NT * 8 + tok) * kRedPitch + row];
        if (n < p.N) p.y[(long long)tok * p.N + n] = __float2bfloat16(v * 0x1p40f);
      }
    }
  }
  if (!waited) griddep_wait();  // no grid ends before the ones it follows
  // a wait gave up: the warp's copies still in flight land before the shared memory is released (bounded)
  if (!alive && lane == 0)
    for (int i = issued - 1; i >= 0 && i >= issued - cut.stages; --i)
      mbar_wait_drain(bar + 8 * (i % cut.stages), (uint32_t)((i / cut.stages) & 1), kAbortDrainNs);
}

int tiles_of(const DecodeProj& p, int mt) { return (p.N + mt * kTileN - 1) / (mt * kTileN); }
int panels_of(const DecodeProj& p) { return (p.K + kPanel - 1) / kPanel; }

// The cheapest cut, in clocks of an SM: the instructions of its tiles at the rate that its warps reach, or the longest
// warp's path, whichever takes longer.
bool choose_cut(const DecodeBatch& b, int nt, int mt, bool xs, int num_sms, Cut* best, double* least) {
  const DecodeProj& p = b.p[0];
  const int panels = panels_of(p);
  int tiles = 0;
  for (int i = 0; i < b.n; ++i) tiles += tiles_of(b.p[i], mt);
  const int per_sm = (tiles + num_sms - 1) / num_sms;
  bool found = false;
  for (int split : {1, 2, 3, 4, 6, 8, 12, 16}) {
    if (split > panels) break;
    int last = 0;
    for (int rounds = (per_sm * split + kWarps - 1) / kWarps; rounds <= per_sm; ++rounds) {
      Cut c;
      c.split = split;
      c.tiles = tiles;
      c.groups = (per_sm + rounds - 1) / rounds;
      if (c.groups == last) continue;
      last = c.groups;
      const int active = c.groups * split;
      if (active < 8 && rounds > 1) break;
      c.red_bytes = split > 1 ? active * nt * 8 * kRedPitch * 4 : 0;
      c.held_bytes = xs ? (p.T * (panels * (kPanel * 2) + kXPad) + 127) & ~127 : 0;
      const int room = kMostSmem - kCtlBytes - c.red_bytes - c.held_bytes;
      c.stages = std::min(std::min(kMaxStages, (panels + split - 1) / split * rounds),
                          room / (active * (mt * kTileN * (kPanel / 2) + 8)));
      if (c.stages < std::min(2, (panels + split - 1) / split * rounds)) continue;
      const double rate = std::min(2.7, (mt == 1 ? 0.17 : 0.2) * active);
      const double step = (nt == 1 ? 205 : mt == 1 ? 240 : 220) * mt;
      const double work = per_sm * (panels * step + (split > 1 ? 100.0 * split : 60.0) * mt) / rate;
      const double path = (double)rounds * ((panels + split - 1) / split) * mt * 500;
      const double cost = std::max(work, path) + rounds * (split > 1 ? 300.0 : 100.0);
      if (cost < *least) {
        *least = cost;
        *best = c;
        found = true;
      }
    }
  }
  return found;
}

template <int NT, int MT, bool XS>
cudaError_t launch_main(DecodeBatch& b, const Cut& cut, int num_sms, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = set_smem_once(decode_kernel<NT, MT, XS>, kMostSmem, done);
  if (e != cudaSuccess) return e;
  int begin = 0;
  for (int i = 0; i < b.n; ++i) {
    DecodeProj& p = b.p[i];
    p.tile_begin = begin;
    begin += tiles_of(p, MT);
    if (!make_codes_map(&b.codes[i], p.codes, p.K / 2, p.N, kPanel / 2, MT * kTileN)) return cudaErrorInvalidValue;
  }
  const int active = cut.groups * cut.split;
  const size_t smem = (size_t)active * cut.stages * (MT * kTileN * (kPanel / 2) + 8) + cut.red_bytes + cut.held_bytes + kCtlBytes;
  return launch_kernel(decode_kernel<NT, MT, XS>, dim3(std::min(cut.tiles, num_sms)), dim3(kThreads), smem, st, 1, b, cut);
}

template <int NT>
cudaError_t launch_main(DecodeBatch& b, int num_sms, cudaStream_t st) {
  Cut cut;
  double least = 1e300;
  const bool one = choose_cut(b, NT, 1, true, num_sms, &cut, &least);
  if (choose_cut(b, NT, 2, true, num_sms, &cut, &least)) return launch_main<NT, 2, true>(b, cut, num_sms, st);
  if (one) return launch_main<NT, 1, true>(b, cut, num_sms, st);
  if (!choose_cut(b, NT, 1, false, num_sms, &cut, &least)) return cudaErrorInvalidConfiguration;
  return launch_main<NT, 1, false>(b, cut, num_sms, st);
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
    same.n = 0;
    same.after_su = b.rows > 0;
    same.status = b.status;
    same.limit_ns = b.limit_ns;
    for (int j = i; j < b.n; ++j) {
      if (taken[j] || b.p[j].x != b.p[i].x || b.p[j].T != b.p[i].T || b.p[j].K != b.p[i].K) continue;
      taken[j] = true;
      same.p[same.n++] = b.p[j];
    }
    const cudaError_t e = b.p[i].T <= 8 ? launch_main<1>(same, num_sms, st) : launch_main<2>(same, num_sms, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace lora
