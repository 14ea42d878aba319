// The few-token forward's second launch for projections of many rows, on the 5th-generation tensor cores:
//   y^T [128 rows, 16 tokens] = W [128, K] . x^T, W the A operand in tensor memory, x the B operand in shared memory
//
// mma.sync takes 24 clocks of a sub-core for 16 x 8 x 16 (measured: 16 tokens cost 64 us on 128256 x 3072 however the
// loads were arranged), so that 9 to 16 tokens are bound by it at twice the time that the weights' bytes take, and
// the activation's fragments fill shared memory's bandwidth.  Here a thread has a row of W: it dequantizes the row's
// codes in order (the same 9 instructions per 8 codes) and stores them into its lane of tensor memory, where a lane
// is a row and a column a pair of K; nothing crosses lanes and no dequantized weight touches shared memory.
//   warp 0       copies: a stage holds 128 rows x 256 columns of codes, and the activation's 256 columns
//   warp 1       issues the MMAs: 16 per panel, N = 16 tokens (zeros past T)
//   warps 4-7    epilogue: a tile's sums to y
//   warps 8-19   three groups that dequantize every third panel each, into a buffer of their own
// The adapter is one more step of a tile: the group's threads store their rows of B, and the stage holds su's three
// terms as the MMAs' B operand.
// A call whose tiles are fewer than the SMs has clusters of CTAs share a tile's columns; their sums meet in the first
// one's shared memory (plan_wide).
// 16 tokens, 128256 x 3072, 222 MB: 45 us, 4.9 TB/s, bound by the dequantization's instructions and the hand-over of the
// panels (each costs the MMAs some 200 clocks; handing a panel over in two or four parts takes 50 and 70 us).
#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace lora {
namespace {

constexpr int kRows = 128, kPanel = 256, kTok = 16;
constexpr int kGroups = 3;  // of warps that dequantize, each with a panel in tensor memory
constexpr int kThreads = 32 * (8 + 4 * kGroups);
constexpr uint32_t kCodeBytes = kRows * kPanel / 2, kXBlock = kTok * 128, kXBytes = kPanel / 64 * kXBlock;
constexpr uint32_t kBufCols = kPanel / 2;  // 32-bit columns of a panel
constexpr uint32_t kDCol = kGroups * kBufCols, kTmemCols = 512;  // behind them the sums of two tiles
constexpr int kMaxStages = 9;
constexpr long long kDrainNs = 100000000ll;
constexpr int kMostSmem = 227 * 1024;
constexpr uint32_t kSumBytes = kTok * kRows * 4;  // of a CTA's sums of a tile
constexpr int kMostSplit = 8;

struct Ctl {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t afull[kGroups], aempty[kGroups];
  uint64_t dfull[2], dempty[2];
  uint64_t drain;
  uint32_t tmem;
  int abort;
};

// D [tmem] (+)= A [tmem] . B [smem]: 128 rows, bf16 inputs, fp32 sums.
__device__ __forceinline__ void umma_bf16_ta(uint32_t d, uint32_t a, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]));
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int CAP>
struct CodeMaps {
  CUtensorMap codes[CAP];
};

struct Wide {
  int tiles, stages;
  int held;   // bytes of the activation (a CTA's columns) that stay in shared memory; 0: a stage carries its columns
  int split;  // CTAs of a cluster that share a tile's columns (then one tile per cluster)
};

template <typename Table>
__global__ void __launch_bounds__(kThreads, 1) decode_wide_kernel(const __grid_constant__ Table b,
                                                                  const __grid_constant__ CodeMaps<Table::kCap> maps,
                                                                  const __grid_constant__ CUtensorMap x_map,
                                                                  const __grid_constant__ Wide wide) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int T = b.p[0].T, K = b.p[0].K, pairs = K / 64;
  // the CTA's tiles, and its panels of them, the c0-th on; the adapter is the first CTA's, whose share is the smallest
  const int split = wide.split, rank = (int)blockIdx.x % split;
  const int tile0 = (int)blockIdx.x / split, stride = (int)gridDim.x / split;
  const int all = (K + kPanel - 1) / kPanel, c0 = all * rank / split, panels = all * (rank + 1) / split - c0;
  const uint32_t stage_bytes = kCodeBytes + (wide.held ? 0u : kXBytes);
  const uint32_t ring = smem_u32(smem), held = ring + wide.stages * stage_bytes;
  uint8_t* rest = smem + wide.stages * stage_bytes + wide.held;
  float* sums = reinterpret_cast<float*>(rest);  // [split][tokens][rows], the first CTA's: the others' sums come here
  Ctl* ctl = reinterpret_cast<Ctl*>(rest + (split > 1 ? split * kSumBytes : 0u));
  volatile int* abort = &ctl->abort;
  const WaitCtl wait{b.status, b.limit_ns};
  const uint32_t full = smem_u32(ctl->full), empty = smem_u32(ctl->empty), afull = smem_u32(ctl->afull);
  const uint32_t aempty = smem_u32(ctl->aempty), dfull = smem_u32(ctl->dfull), dempty = smem_u32(ctl->dempty);

  if (threadIdx.x == 0) {
    for (int i = 0; i < wide.stages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 5);  // the group's warps, and the MMAs on its panel
    }
    for (int i = 0; i < kGroups; ++i) {
      mbar_init(afull + 8 * i, 4);
      mbar_init(aempty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(dfull + 8 * i, 1);
      mbar_init(dempty + 8 * i, 4);
    }
    mbar_init(smem_u32(&ctl->drain), 1);
    ctl->abort = 0;
    fence_mbar_init();
  }
  // not after a launch of this call: tensor memory is taken once the grid before is done
  if (!b.after_su) griddep_wait();
  if (warp == 1) {
    tmem_alloc(smem_u32(&ctl->tmem), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (split > 1) cluster_sync_all();  // every CTA has begun: its shared memory may be written
  griddep_launch_dependents();
  const uint32_t tmem = ctl->tmem;
  long long issued = 0;     // producer: stages
  bool issued_any = false;  // MMAs

  // Stage `it` of the CTA's sequence of panels lies in slot it % stages and is dequantized by group it % kGroups; the
  // ring's length is a multiple of kGroups, so that every wait of a thread follows the slot's fills one by one.
  if (warp == 0) {  // -------------------------------------------------------- copies
    int s = 0, proj = 0;
    uint32_t phase = 1;
    bool ok = true, first = true, waited = !b.after_su;
    auto claim = [&]() { return ok = ok && __all_sync(0xffffffffu, mbar_wait(empty + 8 * s, phase, wait, abort)); };
    auto next = [&]() {
      __syncwarp();
      ++issued;
      if (++s == wide.stages) {
        s = 0;
        phase ^= 1u;
      }
    };
    for (int tile = tile0; tile < wide.tiles && ok; tile += stride, first = false) {
      while (proj + 1 < b.n && tile >= b.p[proj + 1].tile_begin) ++proj;
      const DecodeProj& p = b.p[proj];
      const int n0 = (tile - p.tile_begin) * kRows;
      for (int c = 0; c < panels && claim(); ++c, next()) {
        if (elect_one()) {
          const uint32_t at = ring + s * stage_bytes, bar = full + 8 * s;
          const bool with_x = !wide.held || first;  // the held activation comes with the first tile's codes
          mbar_arrive_expect_tx(bar, kCodeBytes + (with_x ? kXBytes : 0u));
          tma_load_2d(at, &maps.codes[proj], bar, (c0 + c) * (kPanel / 2), n0);
          if (with_x)
            for (int i = 0; i < kPanel / 64; ++i)
              tma_load_2d((wide.held ? held + c * kXBytes : at + kCodeBytes) + i * kXBlock, &x_map, bar,
                          (c0 + c) * kPanel + 64 * i, 0);
        }
      }
      if (p.r > 0 && rank == 0 && claim()) {
        if (!waited) {
          griddep_wait();  // su
          waited = true;
        }
        if (elect_one()) {
          const uint32_t bytes = (uint32_t)(kSuTerms * su_blocks(p.r)) * kXBlock, bar = full + 8 * s;
          mbar_arrive_expect_tx(bar, bytes);
          bulk_load(ring + s * stage_bytes, p.su_image, bytes, bar);
        }
        next();
      }
    }
    if (!waited) griddep_wait();  // no grid ends before the ones it follows
  } else if (warp == 1) {  // ------------------------------------------------- MMAs
    // (the whole warp, converged, one elected lane issuing: the MMAs then take their operands from uniform registers;
    // one thread issuing them took 100 clocks for each)
    constexpr uint32_t idesc = idesc_bf16_f32(kRows, kTok, 0, 0);
    auto wait_all = [&](uint32_t bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_wait(bar, parity, wait, abort));
    };
    int s = 0, group = 0, n = 0, proj = 0;
    uint32_t phase = 0, aphase = 0;  // aphase: of the groups from `group` on
    bool ok = true;
    const uint64_t desc_x = sw128_desc(wide.held ? held : ring + kCodeBytes, 16, 1024);
    auto ready = [&]() {  // the stage's part of shared memory, and the group's of tensor memory
      ok = ok && wait_all(full + 8 * s, phase) && wait_all(afull + 8 * group, aphase);
      tc_fence_after();
      return ok;
    };
    auto release = [&]() {  // by the elected lane
      umma_commit(aempty + 8 * group);
      umma_commit(empty + 8 * s);
    };
    auto next = [&]() {
      __syncwarp();
      issued_any = true;
      if (++s == wide.stages) {
        s = 0;
        phase ^= 1u;
      }
      if (++group == kGroups) {
        group = 0;
        aphase ^= 1u;
      }
    };
    for (int tile = tile0; tile < wide.tiles && ok; tile += stride, ++n) {
      while (proj + 1 < b.n && tile >= b.p[proj + 1].tile_begin) ++proj;
      const int d = n & 1, r = rank == 0 ? b.p[proj].r : 0;
      if (!wait_all(dempty + 8 * d, (uint32_t)((n >> 1) & 1) ^ 1u)) break;
      tc_fence_after();
      const uint32_t d_tmem = tmem + kDCol + (uint32_t)(d * kTok);
      for (int c = 0; c < panels && ready(); ++c, next()) {
        const uint64_t bd = desc_x + ((wide.held ? (uint32_t)c * kXBytes : (uint32_t)s * stage_bytes) >> 4);
        const uint32_t a_tmem = tmem + (uint32_t)group * kBufCols, more = c != 0 ? 1u : 0u;
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < kPanel / 16; ++k)
            umma_bf16_ta(d_tmem, a_tmem + 8 * k, bd + (k / 4) * (kXBlock >> 4) + 2 * (k % 4), idesc, k != 0 ? 1u : more);
          release();
        }
      }
      if (r > 0 && ready()) {  // the adapter: its 16 columns at a time, against each term of su
        const uint64_t su = sw128_desc(ring + (uint32_t)s * stage_bytes, 16, 1024);
        const uint32_t a_tmem = tmem + (uint32_t)group * kBufCols;
        if (elect_one()) {
          for (int e = 0; e < kSuTerms; ++e)
            for (int k = 0; k < su_steps(r); ++k)
              umma_bf16_ta(d_tmem, a_tmem + 8 * k,
                           su + (uint32_t)(e * su_blocks(r) + k / 4) * (kXBlock >> 4) + 2 * (k % 4), idesc, 1u);
          release();
        }
        next();
      }
      if (ok && elect_one()) umma_commit(dfull + 8 * d);
      __syncwarp();
    }
  } else if (warp >= 4 && warp < 8) {  // ------------------------------------- epilogue
    const int q = warp & 3;
    int proj = 0, n = 0;
    for (int tile = tile0; tile < wide.tiles; tile += stride, ++n) {
      while (proj + 1 < b.n && tile >= b.p[proj + 1].tile_begin) ++proj;
      const DecodeProj& p = b.p[proj];
      const int d = n & 1, row = (tile - p.tile_begin) * kRows + q * 32 + lane;
      if (!mbar_wait(dfull + 8 * d, (uint32_t)((n >> 1) & 1), wait, abort)) break;
      __syncwarp();
      tc_fence_after();
      uint32_t v[16];
      tmem_ld_32x32b_x16(tmem + ((uint32_t)(q * 32) << 16) + kDCol + d * kTok, v);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(dempty + 8 * d);
      if (split > 1) {
        const uint32_t to = mapa_shared(smem_u32(sums), 0) + (uint32_t)rank * kSumBytes + (uint32_t)(q * 32 + lane) * 4u;
#pragma unroll
        for (int e = 0; e < kTok; ++e)
          if (e < T) st_cluster_u32(to + (uint32_t)(e * kRows) * 4u, v[e]);
      } else if (row < p.N) {
#pragma unroll
        for (int e = 0; e < kTok; ++e)
          if (e < T) p.y[(long long)e * p.N + row] = __float2bfloat16(__uint_as_float(v[e]) * 0x1p40f);
      }
    }
  } else if (warp >= 8) {  // ------------------------------------------------- dequantization
    const int group = (warp - 8) / 4, q = warp & 3, row = q * 32 + lane;
    // the group's next step: panel c of a tile (c == panels: the adapter), and its (s, b) pairs, loaded a step ahead
    int tile = tile0, c = group, proj = 0, steps = 0;
    const uint32_t* pair_at = nullptr;
    const __nv_bfloat16* adapter = nullptr;  // the row's
    bool in_row = false;
    auto open = [&]() {
      if (tile >= wide.tiles) return;
      while (proj + 1 < b.n && tile >= b.p[proj + 1].tile_begin) ++proj;
      const DecodeProj& p = b.p[proj];
      const int n = (tile - p.tile_begin) * kRows + row;
      steps = panels + (p.r > 0 && rank == 0);
      in_row = n < p.N;
      pair_at = reinterpret_cast<const uint32_t*>(p.params) + (long long)n * pairs;
      adapter = p.B + (long long)n * p.r;
    };
    auto settle = [&]() {
      while (tile < wide.tiles && c >= steps) {
        c -= steps;
        tile += stride;
        open();
      }
    };
    uint32_t next[4];
    auto fetch = [&]() {
      if (tile >= wide.tiles || c == panels) return;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 4 * (c0 + c) + i;
        next[i] = in_row && at < pairs ? __ldg(pair_at + at) : 0u;
      }
    };
    open();
    settle();
    fetch();
    int s = group;
    uint32_t phase = 0, aphase = 1;
    const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16) + group * kBufCols;
    auto advance = [&]() {
      c += kGroups;
      settle();
      fetch();
    };
    auto buffer_free = [&]() {  // the MMAs on the group's step before are done
      const bool ok = __all_sync(0xffffffffu, mbar_wait(aempty + 8 * group, aphase, wait, abort));
      tc_fence_after();
      return ok;
    };
    while (tile < wide.tiles) {
      if (c == panels) {  // the adapter's row, 32 columns at a time, zeros behind column r
        const int r = b.p[proj].r;
        const uint16_t* B = reinterpret_cast<const uint16_t*>(in_row ? adapter : nullptr);
        advance();
        if (!buffer_free()) break;
        for (int j0 = 0; j0 < r; j0 += 32) {
          uint32_t o[16];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = j0 + 8 * i;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (B && r % 8 == 0 && j < r) {
              v = __ldg(reinterpret_cast<const uint4*>(B + j));
            } else if (B) {
              uint32_t h[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) h[e] = j + e < r ? __ldg(B + j + e) : 0u;
              v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
            }
            o[4 * i] = v.x;
            o[4 * i + 1] = v.y;
            o[4 * i + 2] = v.z;
            o[4 * i + 3] = v.w;
          }
          __syncwarp();
          tmem_st_32x32b_x16(lanes + j0 / 2, o);
        }
        // the slot's fills are followed one by one, also this one, which is for the MMAs
        if (!__all_sync(0xffffffffu, mbar_wait(full + 8 * s, phase, wait, abort))) break;
      } else {
        uint32_t s0[4], s1[4], of[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t sb = dq40_pair(next[i]);
          s0[i] = __byte_perm(sb, 0u, 0x1010);
          of[i] = __byte_perm(sb, 0u, 0x3232);
          s1[i] = dq40_high(s0[i]);
        }
        advance();
        if (!__all_sync(0xffffffffu, mbar_wait(full + 8 * s, phase, wait, abort))) break;
        const uint8_t* codes = smem + s * stage_bytes + row * (kPanel / 2);
        uint4 w4[2];  // of 32 codes each
        auto load = [&](int i) {  // the 64 codes of pair i
#pragma unroll
          for (int u = 0; u < 2; ++u)
            w4[u] = *reinterpret_cast<const uint4*>(codes + (((2 * i + u) ^ (row & 7)) * 16));
        };
        load(0);
        bool ok = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t o[2][16];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t w[4] = {w4[u].x, w4[u].y, w4[u].z, w4[u].w};
#pragma unroll
            for (int m = 0; m < 4; ++m)
              dq40_word(w[m], s0[i], s1[i], of[i], o[u][4 * m], o[u][4 * m + 1], o[u][4 * m + 2], o[u][4 * m + 3]);
          }
          if (i < 3) load(i + 1);
          if (i == 0 && !(ok = buffer_free())) break;
#pragma unroll
          for (int u = 0; u < 2; ++u) tmem_st_32x32b_x16(lanes + 32 * i + 16 * u, o[u]);
        }
        if (!ok) break;
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(empty + 8 * s);
        mbar_arrive(afull + 8 * group);
      }
      s += kGroups;
      if (s >= wide.stages) {
        s = group;
        phase ^= 1u;
      }
      aphase ^= 1u;
    }
  }

  if (split > 1) {  // ------------------------------------------------------- the cluster's sums, in the order of its CTAs
    __syncwarp();
    cluster_sync_all();
    if (rank == 0) {
      int proj = 0;
      while (proj + 1 < b.n && tile0 >= b.p[proj + 1].tile_begin) ++proj;
      const DecodeProj& p = b.p[proj];
      const int n0 = (tile0 - p.tile_begin) * kRows, rows = min(kRows, p.N - n0);
      for (int o = threadIdx.x; o < kRows * T; o += kThreads) {
        const int e = o / kRows, i = o % kRows;
        if (i >= rows) continue;
        float v = 0.f;
        for (int k = 0; k < split; ++k) v += sums[(k * kTok + e) * kRows + i];
        p.y[(long long)e * p.N + n0 + i] = __float2bfloat16(v * 0x1p40f);
      }
    }
  }

  // ------------------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (*abort) {
    // a wait gave up: this CTA's copies and MMAs complete before its memory is released (bounded)
    if (warp == 0 && lane == 0)
      for (long long i = std::max(0ll, issued - wide.stages); i < issued; ++i)
        mbar_wait_drain(full + 8 * (uint32_t)(i % wide.stages), (uint32_t)((i / wide.stages) & 1), kDrainNs);
    if (warp == 1 && lane == 0 && issued_any) {
      umma_commit(smem_u32(&ctl->drain));
      mbar_wait_drain(smem_u32(&ctl->drain), 0, kDrainNs);
    }
    tc_fence_before();
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace

namespace {

// Clusters of `ctas` CTAs that run at once: one CTA per SM, a cluster within one of the GPU's groups of SMs.
int most_clusters(int ctas) {
  static std::atomic<int> cache[64][kMostSplit + 1];  // 0: not asked yet
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  std::atomic<int>& known = cache[dev & 63][ctas];
  int n = known.load(std::memory_order_relaxed);
  if (n) return n;
  static std::atomic<unsigned long long> done{0};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kMostSmem;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)ctas;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (set_smem_once(decode_wide_kernel<DecodeTable<8>>, kMostSmem, done) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, decode_wide_kernel<DecodeTable<8>>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  known.store(std::max(n, 1), std::memory_order_relaxed);
  return n;
}

}  // namespace

// The launch starts late (tensor memory, the first panels), each step of a CTA, a panel or the adapter, takes 0.475 us
// whatever the tokens, and the adapter waits for the launch before.  Where tiles leave SMs idle, the CTAs of a cluster
// share a tile's panels.  (Alone and shared: 8192 x 8192, r 16, 16 tokens, 20.8 and 15.7 us by two; 8192 x 3072 20.3 and
// 11.7 by five; 5120 rows of 3072 11.0 and 9.7 by three; six for 3072 rows, one cluster more than run at once, 18.8.)
WidePlan plan_wide(long long tiles, int panels, int rank, int num_sms) {
  const int adapter = rank > 0;
  const double late = adapter * 1.6 + 0.02 * rank;
  WidePlan best{1, 4.6 + late + (double)((tiles + num_sms - 1) / num_sms) * (panels + adapter) * 0.475};
  for (int s = 2; s <= kMostSplit && s <= panels; ++s) {
    const double us = 4.9 + late + 0.8 * adapter + std::max((panels + s - 1) / s, panels / s + adapter) * 0.475;
    if (us < best.us && tiles <= num_sms / s && tiles <= most_clusters(s)) best = WidePlan{s, us};
  }
  return best;
}

cudaError_t launch_decode_wide(DecodeBatch& b, int num_sms, cudaStream_t st) {
  const DecodeProj& p0 = b.p[0];
  const int panels = (p0.K + kPanel - 1) / kPanel;
  Wide w;
  w.tiles = 0;
  int rank = 0;
  for (int i = 0; i < b.n; ++i) {
    rank = std::max(rank, b.p[i].r);
    b.p[i].tile_begin = w.tiles;
    w.tiles += (b.p[i].N + kRows - 1) / kRows;
  }
  CUtensorMap x_map;
  if (!make_bf16_map(&x_map, p0.x, p0.K, p0.T, 64, kTok)) return cudaErrorInvalidValue;
  w.split = plan_wide(w.tiles, panels, rank, num_sms).split;
  // the activation is held where at least two stages of codes per group fit beside it
  const int sums = w.split > 1 ? w.split * (int)kSumBytes : 0, room = kMostSmem - (int)sizeof(Ctl) - sums;
  const int all = (panels + w.split - 1) / w.split * (int)kXBytes;
  w.held = all + 2 * kGroups * (int)kCodeBytes <= room ? all : 0;
  const int stage = kCodeBytes + (w.held ? 0 : kXBytes);
  w.stages = std::min(kMaxStages, (room - w.held) / stage) / kGroups * kGroups;
  const size_t smem = (size_t)w.stages * stage + w.held + sums + sizeof(Ctl);
  const int ctas = w.split > 1 ? w.tiles * w.split : std::min(w.tiles, num_sms);
  return with_table(b, [&](const auto& t) {
    using Table = std::decay_t<decltype(t)>;
    CodeMaps<Table::kCap> maps;
    for (int i = 0; i < t.n; ++i)
      if (!make_bytes_map(&maps.codes[i], t.p[i].codes, t.p[i].K / 2, t.p[i].N, kPanel / 2, kRows))
        return cudaErrorInvalidValue;
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = set_smem_once(decode_wide_kernel<Table>, kMostSmem, done);
    if (e != cudaSuccess) return e;
    return launch_kernel(decode_wide_kernel<Table>, dim3(ctas), dim3(kThreads), smem, st, w.split, t, maps, x_map, w);
  });
}

}  // namespace lora
