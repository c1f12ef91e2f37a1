// Block-scaled products grouped by expert: rows of E4M3 codes lie in the order of the experts, expert e's at offsets[e] .. offsets[e+1] - 1, and each
// meets the weights of its own.  The offsets are read on the GPU, so that a router's answer need not reach the host.
//
//   experts_pair_kernel    C[t, n] = sum_k X(t, k) W_e(n, k), e the expert of row t: forward products, and input gradients, which sum over the stored rows of W_e
//   experts_rows_kernel    the same where experts have few rows and reading W is what costs: 128 lines of W and 16 to 64 rows a tile, clusters along K
//   segments_pair_kernel   C_e[m, n] = sum over the rows t of e of A(t, m) B(t, n): weight gradients
//
// UE8M0 scales, applied by the tensor cores (tcgen05.mma kind::mxf8f6f4), as in the product with one matrix; pairs of CTAs with the TMA producer, the MMA issuer,
// the scale writers and the epilogue in warps of their own take tiles one after another.
//
// In experts_pair_kernel the WEIGHTS' lines are the 256 rows of the instruction and the tokens its columns, 32 to 224 of them: a segment of any length is
// divided into tiles of nearly equal width, so that a short one costs what it holds and not a tile of 256.  Two accumulators of 224 columns and the scale words fit tensor
// memory side by side.  Results leave row by row of C, 64 bytes a warp, BF16 ones in pieces of 16 bytes a lane by way of shared memory (K = 500: 71 us, pairs of columns from
// registers 118; level from K = 2048 on): no row of another segment is touched.
// Measured in bursts: 16384 rows of 16 uneven experts, 4096 -> 4096, 240 us (2.3 PFLOP/s; twelve equal ones 2.5, the product with one matrix 2.8), bound by the tensor cores, by
// the traffic of narrower tiles, and back to back by the power limit (280 us); 9001 rows of 24 experts, 2048 -> 4096, 92 us, and 131 us where the
// weights' rows are not whole 128-byte lines (2056).  244 rows of 32 experts, 4096 -> 2048, 47 us (5.0 TB/s, memory).  Weight gradients of 16 experts, 4096 x 2048 from 16384
// rows, added in FP32: 234 us (5.0 TB/s, memory: the sums are read and written).
#include <type_traits>

#include "ozk_fp8_product.cuh"
#include "ozk_wait.cuh"

namespace ozk {
namespace {

constexpr int kTokens = 224;        // most rows of C in a tile
constexpr int kTokenStep = 32;      // widths of the instruction on a pair of CTAs
constexpr int kLines = 256;         // lines of the weights in a tile
constexpr int kMostExperts = 1024;  // the table of segments lies in shared memory
constexpr int kGroupBand = 16;      // tiles of a segment that sweep the weights together
constexpr int kXBoxes = 4;          // heights of the boxes of X: half a tile's width, rounded up to one of these
__host__ __device__ constexpr int x_box(int i) { return i == 0 ? 16 : i == 1 ? 32 : i == 2 ? 64 : 112; }
__device__ __forceinline__ int x_box_of(int half) { return half <= 16 ? 0 : half <= 32 ? 1 : half <= 64 ? 2 : 3; }

struct __align__(64) ExpertMaps {
  CUtensorMap w, x[kXBoxes];
};
struct ExpertParams {
  Operand x, w;            // w: one expert's
  int64_t w_scale_step;    // from one expert's scales to the next
  const int* offsets;
  int experts, rows;
  void* out;
  int64_t ldc;
  int N, tiles_n, groups;
  int chunk;               // blocks summed in tensor memory before the sum is added to C in FP32, a multiple of 4
  int pairs_ok, wide_ok, pieces_ok;   // BF16 results may be stored two, four or eight at a time
  int clear;               // rows outside the segments become zero
  StatusBlock* status;
};

constexpr int kPairStages = 6;
struct __align__(8) ExpertShared {
  uint64_t full[kPairStages], empty[kPairStages];
  uint64_t sf_full[2], sf_empty[2];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t overlap, drained;
  uint32_t tmem_base;
  volatile int abort;
};
static_assert(sizeof(ExpertShared) <= 512, "room reserved behind the stages");

constexpr int kFirstEpilogue = 6, kEpilogueWarps = 8, kPairThreads = 32 * (kFirstEpilogue + kEpilogueWarps);
constexpr int kScaleCol = 480;   // two sets of 4 columns for one operand, 8 for the other
struct ExpertShape {
  static constexpr int kWBytes = 128 * kBlock, kXBytes = kTokens / 2 * kBlock;
  static constexpr int kStageBytes = kWBytes + kXBytes;
  static constexpr int kStaging = kEpilogueWarps * 2048;   // 32 rows of 32 BF16 results a warp
  static size_t smem(int experts) { return (size_t)kPairStages * kStageBytes + kStaging + 512 + (size_t)(3 * experts + 1) * 4 + 1024; }
};

// The table of segments: where each begins and ends, and how many tiles of at most kTokens rows lie before it.  By one warp.  Offsets are held within the
// rows and never fall, so that whatever they are no row belongs to two segments.
__device__ __forceinline__ void segment_table(const int* offsets, int experts, int rows, int lane, int* begin, int* end, int* before) {
  int carry = 0, top = min(max(__ldg(offsets), 0), rows);
  for (int e0 = 0; e0 < experts; e0 += 32) {
    const int e = e0 + lane;
    int f = e < experts ? min(max(__ldg(offsets + e + 1), top), rows) : top;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, f, d);
      if (lane >= d) f = max(f, v);
    }
    int b = __shfl_up_sync(0xFFFFFFFFu, f, 1);
    if (lane == 0) b = top;
    const int u = (f - b + kTokens - 1) / kTokens;
    int sum = u;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, sum, d);
      if (lane >= d) sum += v;
    }
    if (e < experts) begin[e] = b, end[e] = f, before[e] = carry + sum - u;
    carry += __shfl_sync(0xFFFFFFFFu, sum, 31);
    top = __shfl_sync(0xFFFFFFFFu, f, 31);
  }
  if (lane == 0) before[experts] = carry;
}

struct ExpertItem {
  int expert, n0, t0, count, width, box;   // `count` rows from t0 on, in an instruction of `width` columns
};
// Items in the order of the experts; in an expert, bands of kGroupBand tiles of its rows sweep the lines, so that pairs at work together share panels.
struct ExpertWalk {
  const int *begin, *end, *before;
  int tiles_n, expert = 0;
  __device__ __forceinline__ ExpertItem at(int item) {
    const int unit = item / tiles_n;
    while (before[expert + 1] <= unit) ++expert;
    const int rows = end[expert] - begin[expert], tiles = before[expert + 1] - before[expert];
    const int width = ((rows + tiles - 1) / tiles + kTokenStep - 1) / kTokenStep * kTokenStep;
    const int rem = item - before[expert] * tiles_n, band = kGroupBand * tiles_n, g = rem / band, r = rem - g * band;
    const int in_band = min(kGroupBand, tiles - kGroupBand * g), tile = kGroupBand * g + r % in_band;
    ExpertItem it;
    it.expert = expert;
    it.n0 = r / in_band * kLines;
    it.t0 = begin[expert] + tile * width;
    it.count = min(width, rows - tile * width);
    it.width = (it.count + kTokenStep - 1) / kTokenStep * kTokenStep;
    it.box = x_box_of(it.width / 2);
    return it;
  }
};

// Copies in flight land before a CTA that gave up leaves.
__device__ __forceinline__ void drain_copies(uint64_t* full, int issued) {
  const uint64_t t0 = global_timer_ns();
  for (int j = max(0, issued - kPairStages); j < issued; ++j)
    while (!mbar_try_wait(smem_u32(&full[j % kPairStages]), (uint32_t)(j / kPairStages) & 1u) && global_timer_ns() - t0 < kWaitLimitNs) {
    }
}
__device__ __forceinline__ void drain_products(uint64_t* drained) {
  mma_commit_pair(smem_u32(drained), (uint16_t)1);
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(smem_u32(drained), 0u) && global_timer_ns() - t0 < kWaitLimitNs) {
  }
}
__device__ __forceinline__ void init_barriers(ExpertShared* sh) {
  for (int s = 0; s < kPairStages; ++s) mbar_init(smem_u32(&sh->full[s]), 1), mbar_init(smem_u32(&sh->empty[s]), 1);   // full: the leader's only
  for (int s = 0; s < 2; ++s) mbar_init(smem_u32(&sh->sf_full[s]), 8), mbar_init(smem_u32(&sh->sf_empty[s]), 1);      // 4 scale warps of each CTA
  for (int s = 0; s < 2; ++s) mbar_init(smem_u32(&sh->acc_full[s]), 1), mbar_init(smem_u32(&sh->acc_empty[s]), 2 * kEpilogueWarps);
  mbar_init(smem_u32(&sh->overlap), 8);
  mbar_init(smem_u32(&sh->drained), 1);
  sh->abort = 0;
  fence_barrier_init();
  fence_proxy_async();
}

template <bool kBf16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
experts_pair_kernel(const __grid_constant__ ExpertMaps maps, const __grid_constant__ ExpertParams p) {
  using S = ExpertShape;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* staging = tiles + kPairStages * S::kStageBytes;
  ExpertShared* sh = reinterpret_cast<ExpertShared*>(staging + S::kStaging);
  int* before = reinterpret_cast<int*>(staging + S::kStaging + 512);
  int *begin = before + p.experts + 1, *end = begin + p.experts;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    prefetch_tensormap(&maps.w);
    for (int i = 0; i < kXBoxes; ++i) prefetch_tensormap(&maps.x[i]);
    init_barriers(sh);
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&sh->tmem_base), 512);
    tmem_relinquish_pair();
  }
  if (warp == 2) segment_table(p.offsets, p.experts, p.rows, lane, begin, end, before);
  tc_fence_before();
  __syncthreads();
  cluster_arrive();   // the peer's barriers are initialised before anything is sent to them
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem = sh->tmem_base;
  const int items = before[p.experts] * p.tiles_n;
  ExpertWalk walk{begin, end, before, p.tiles_n};

  if (warp == 0) {
    // ------------------------------ TMA producer (both CTAs) ------------------------------
    if (lane == 0) {
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int item = pair; item < items && ok; item += npairs) {
        const ExpertItem it = walk.at(item);
        const CUtensorMap* map_x = &maps.x[it.box];
        const uint32_t bytes = 2 * (S::kWBytes + x_box(it.box) * kBlock);
        const int t = it.t0 + rank * (it.width / 2);
        for (int b = 0; b < p.x.blocks; ++b) {
          if (!wait_bounded(smem_u32(&sh->empty[stage]), phase ^ 1u, &sh->abort, p.status, 0xA00 + stage)) {
            ok = false;
            break;
          }
          const uint32_t full = map_to_cta(smem_u32(&sh->full[stage]), 0);
          const uint32_t dst = smem_u32(tiles + stage * S::kStageBytes);
          if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh->full[stage]), bytes);
          int x, y;
          tile_at(p.w.contract_rows, it.n0 + rank * 128, b, x, y);
          tma_load_3d_pair(dst, &maps.w, full, x, y, it.expert);
          tma_load_2d_pair(dst + S::kWBytes, map_x, full, b * kBlock, t);
          ++issued;
          if (++stage == kPairStages) stage = 0, phase ^= 1u;
        }
      }
      if (sh->abort && rank == 0) drain_copies(sh->full, issued);
    }
  } else if (warp == 1) {
    // ------------------------------ MMA issuer (leader only) ------------------------------
    if (rank == 0) {
      int stage = 0;
      uint32_t phase = 0, unit = 0, sf_unit = 0;
      const int w_lines = p.w.contract_rows;
      const uint32_t w_step = operand_step(w_lines), x_step = operand_step(0);
      bool ok = true;
      for (int item = pair; item < items && ok; item += npairs) {
        const ExpertItem it = walk.at(item);
        const uint32_t idesc = idesc_mxf8(kLines, it.width, w_lines, 0);
        for (int b0 = 0; b0 < p.x.blocks && ok; b0 += p.chunk, ++unit) {
          const int b_end = min(p.x.blocks, b0 + p.chunk);
          const uint32_t buf = unit & 1u, acc = tmem + buf * kTokens;
          if (!wait_warp(smem_u32(&sh->acc_empty[buf]), ((unit >> 1) & 1u) ^ 1u, &sh->abort, p.status, 0xA10)) { ok = false; break; }
          tc_fence_after();
          for (int b = b0; b < b_end; ++b) {
            const uint32_t set = sf_unit & 1u, sfa = tmem + kScaleCol + set * 12, sfb = sfa + 4;
            if ((b & 3) == 0 && !wait_warp(smem_u32(&sh->sf_full[set]), (sf_unit >> 1) & 1u, &sh->abort, p.status, 0xA11)) { ok = false; break; }
            if (!wait_warp(smem_u32(&sh->full[stage]), phase, &sh->abort, p.status, 0xA20 + stage)) { ok = false; break; }
            tc_fence_after();
            const uint32_t base = smem_u32(tiles + stage * S::kStageBytes);
            const uint64_t dw = operand_desc(w_lines, base), dx = operand_desc(0, base + S::kWBytes);
            const bool last = b + 1 == b_end, last_of_scales = (b & 3) == 3 || last;
            if (elect_one()) {
#pragma unroll
              for (uint32_t ks = 0; ks < 4; ++ks)
                mma_mxf8_pair(acc, dw + ks * w_step, dx + ks * x_step, idesc | idesc_mxf8_block((uint32_t)b & 3u), sfa, sfb, (b > b0 || ks) ? 1u : 0u);
              mma_commit_pair(smem_u32(&sh->empty[stage]), (uint16_t)3);
              if (last_of_scales) mma_commit_pair(smem_u32(&sh->sf_empty[set]), (uint16_t)3);
              if (last) mma_commit_pair(smem_u32(&sh->acc_full[buf]), (uint16_t)3);
            }
            __syncwarp();
            if (++stage == kPairStages) stage = 0, phase ^= 1u;
            sf_unit += last_of_scales;
          }
        }
      }
      if (sh->abort && elect_one()) drain_products(&sh->drained);
    }
  } else if (warp < kFirstEpilogue) {
    // ------------------------------ scale words into tensor memory (both CTAs) ------------------------------
    // Row r of an operand's 128 lines is lane r % 32, column r / 32 of its four columns, in every quarter of the lanes:
    // each warp writes the quarter it may touch.  This CTA's 128 lines of the weights, all of the tokens.
    const uint32_t at = tmem + (((uint32_t)(warp & 3) * 32u) << 16) + kScaleCol;
    const uint32_t leader = map_to_cta(smem_u32(&sh->sf_full[0]), 0);
    uint32_t unit = 0;
    bool ok = true;
    for (int item = pair; item < items && ok; item += npairs) {
      const ExpertItem it = walk.at(item);
      Operand w = p.w;
      w.scales = static_cast<const uint8_t*>(p.w.scales) + it.expert * p.w_scale_step;
      uint32_t ww[4], wx0[4], wx1[4];   // the words of the next group, on their way while this one's are written
      auto fetch = [&](int g) {
        scale_words<4>(w, it.n0 + rank * 128, lane, g, ww);
        scale_words<4>(p.x, it.t0, lane, g, wx0);
        if (it.width > 128) scale_words<3>(p.x, it.t0 + 128, lane, g, wx1);
      };
      fetch(0);
      for (int g = 0; g < p.groups; ++g, ++unit) {
        const uint32_t set = unit & 1u;
        if (!wait_warp(smem_u32(&sh->sf_empty[set]), ((unit >> 1) & 1u) ^ 1u, &sh->abort, p.status, 0xA30)) {
          ok = false;
          break;
        }
        tc_fence_after();
        tmem_st_32x4(at + set * 12, ww);
        tmem_st_32x4(at + set * 12 + 4, wx0);
        if (it.width > 128) tmem_st_32x4(at + set * 12 + 8, wx1);
        if (g + 1 < p.groups) fetch(g + 1);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(leader + set * 8);
      }
    }
  } else {
    // ------------------------------ epilogue (both CTAs) ----------------------------------
    using T = typename std::conditional<kBf16, uint16_t, float>::type;
    T* out = static_cast<T*>(p.out);
    const uint32_t quad = (uint32_t)(warp & 3);
    const int part = (warp - kFirstEpilogue) >> 2;   // which of the groups of 32 tokens, by turns
    const uint32_t lanes = tmem + ((quad * 32u) << 16);
    const uint32_t empty0 = map_to_cta(smem_u32(&sh->acc_empty[0]), 0);
    if (p.clear) {
      const int first = begin[0], behind = end[p.experts - 1], rest = first + p.rows - behind;
      for (int i = (int)blockIdx.x * kEpilogueWarps + warp - kFirstEpilogue; i < rest; i += (int)gridDim.x * kEpilogueWarps) {
        T* row = out + (int64_t)(i < first ? i : i - first + behind) * p.ldc;
        for (int n = lane; n < p.N; n += 32) row[n] = 0;
      }
    }
    uint32_t unit = 0;
    const int ranges = (p.x.blocks + p.chunk - 1) / p.chunk;
    for (int at = pair * ranges; at < items * ranges; at += at % ranges + 1 < ranges ? 1 : (npairs - 1) * ranges + 1, ++unit) {
      const ExpertItem it = walk.at(at / ranges);
      const bool later = at % ranges != 0;   // a later range of K is added to the earlier ones, by the same thread
      const uint32_t buf = unit & 1u;
      if (!wait_warp(smem_u32(&sh->acc_full[buf]), (unit >> 1) & 1u, &sh->abort, p.status, 0xA40)) break;
      tc_fence_after();
      const int n = it.n0 + rank * 128 + (int)quad * 32 + lane, chunks = it.width / 32;
      for (int c = part; c < chunks; c += 2) {
        uint32_t d[32];
        tmem_ld_32x32(lanes + buf * kTokens + c * 32, d);
        tmem_wait_ld();
        if (c + 2 >= chunks) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(empty0 + buf * 8);
        }
        T* row = out + (int64_t)(it.t0 + c * 32) * p.ldc;
        const int count = it.count - c * 32;   // the same for all lanes
        if constexpr (kBf16) {
          if (p.pieces_ok) {   // through the warp's staging memory: eight columns of one row a lane
            uint32_t* box = reinterpret_cast<uint32_t*>(staging + (warp - kFirstEpilogue) * 2048);
            const int odd = lane & 1, first = n - lane;
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float got = __uint_as_float(__shfl_xor_sync(0xFFFFFFFFu, odd ? d[j] : d[j + 1], 1));
              box[(j + odd) * 16 + lane / 2] = odd ? pack_bf16(got, __uint_as_float(d[j + 1])) : pack_bf16(__uint_as_float(d[j]), got);
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int j = i * 8 + lane / 4, col = first + lane % 4 * 8;
              const uint4 v = *reinterpret_cast<const uint4*>(box + j * 16 + lane % 4 * 4);
              if (j >= count || col >= p.N) continue;
              T* at = row + (int64_t)j * p.ldc + col;
              if (col + 8 <= p.N) {
                *reinterpret_cast<uint4*>(at) = v;
              } else {
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int k = 0; k < 8; ++k)
                  if (col + k < p.N) at[k] = (uint16_t)(w[k / 2] >> (16 * (k % 2)));
              }
            }
            __syncwarp();
            continue;
          }
          if (p.pairs_ok) {   // two columns of one row a lane: even lanes the even rows, odd lanes the odd ones
            const int odd = lane & 1, col = n - odd;
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              if (j >= count) break;
              const float got = __uint_as_float(__shfl_xor_sync(0xFFFFFFFFu, odd ? d[j] : d[j + 1], 1));
              const uint32_t v = odd ? pack_bf16(got, __uint_as_float(d[j + 1])) : pack_bf16(__uint_as_float(d[j]), got);
              if (j + odd < count) {
                T* at = row + (int64_t)(j + odd) * p.ldc + col;
                if (col + 1 < p.N) *reinterpret_cast<uint32_t*>(at) = v; else if (col < p.N) *at = (uint16_t)v;
              }
            }
            continue;
          }
        }
        if (n < p.N) {
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            if (j >= count) break;
            T* at = row + (int64_t)j * p.ldc + n;
            if constexpr (kBf16) *at = (uint16_t)pack_bf16(__uint_as_float(d[j]), 0.f); else *at = later ? *at + __uint_as_float(d[j]) : __uint_as_float(d[j]);
          }
        }
      }
      if (part >= chunks && lane == 0) mbar_arrive_cluster(empty0 + buf * 8);   // 32 tokens: nothing to read for the second half
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_arrive();   // neither CTA leaves while the other may still signal its barriers
  cluster_wait();
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc_pair(tmem, 512);
  }
}

// ---- few rows an expert -----------------------------------------------------------------
// Which tile of a segment this is: its expert, first row and rows (count = 0: there is none), and the rows that segments cover.
struct RowsTile {
  int expert, t0, count, first, behind;
};
// By one warp, each lane with a run of consecutive experts: offsets are held within the rows and never fall.
__device__ __forceinline__ RowsTile rows_tile(const int* offsets, int experts, int rows, int tile, int height, int lane) {
  const int per = (experts + 31) / 32, e0 = min(lane * per, experts), e1 = min(e0 + per, experts);
  const int first = min(max(__ldg(offsets), 0), rows);
  int top = first;   // largest offset up to the end of this lane's run
  for (int e = e0; e < e1; ++e) top = max(top, min(__ldg(offsets + e + 1), rows));
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int v = __shfl_up_sync(0xFFFFFFFFu, top, d);
    if (lane >= d) top = max(top, v);
  }
  const int behind = __shfl_sync(0xFFFFFFFFu, top, 31);
  int before = __shfl_up_sync(0xFFFFFFFFu, top, 1);   // where this lane's run begins
  if (lane == 0) before = first;
  int tiles = 0;
  for (int e = e0, b = before; e < e1; ++e) {
    const int f = max(b, min(__ldg(offsets + e + 1), rows));
    tiles += (f - b + height - 1) / height;
    b = f;
  }
  int sum = tiles;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int v = __shfl_up_sync(0xFFFFFFFFu, sum, d);
    if (lane >= d) sum += v;
  }
  RowsTile r{0, 0, 0, first, behind};
  const uint32_t beyond = __ballot_sync(0xFFFFFFFFu, tile < sum);
  if (!beyond) return r;
  const int l = __ffs(beyond) - 1;
  int left = tile - (sum - tiles);   // in this lane's run, if it is lane l's
  if (lane == l) {
    for (int e = e0, b = before; e < e1; ++e) {
      const int f = max(b, min(__ldg(offsets + e + 1), rows)), n = (f - b + height - 1) / height;
      if (left < n) {
        r.expert = e, r.t0 = b + left * height, r.count = min(height, f - r.t0);
        break;
      }
      left -= n;
      b = f;
    }
  }
  r.expert = __shfl_sync(0xFFFFFFFFu, r.expert, l), r.t0 = __shfl_sync(0xFFFFFFFFu, r.t0, l), r.count = __shfl_sync(0xFFFFFFFFu, r.count, l);
  return r;
}

constexpr int kRowsThreads = 6 * 32;   // producer, issuer, 4 warps for scales and epilogue
constexpr int kRowsMostCluster = 8;
constexpr int kRowsRange = 8;          // groups summed by the tensor cores alone where the result is FP32
template <int NT>
struct ExpertRowsShape {
  static constexpr int kWBytes = 128 * kBlock, kStageBytes = kWBytes + NT * kBlock, kStages = 4, kSets = 4;
  static constexpr int kCols = NT + kSets * 8 <= 64 ? 64 : 128;
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 512 + 1024;
  static_assert(NT * 128 * 4 <= kStages * kStageBytes, "the partial sums are exchanged in the stages' memory");
};
struct __align__(8) ExpertRowsShared {
  uint64_t full[4], empty[4], sf_full[4], sf_empty[4], acc_full, drained;
  uint32_t tmem_base;
  volatile int abort;
  RowsTile tile;
};
static_assert(sizeof(ExpertRowsShared) <= 512, "room reserved behind the stages");

__device__ __forceinline__ float4 load_cluster_f32x4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}

// The lines of W are the instruction's 128 rows, NT rows of C its columns.  The CTAs of a cluster share K and add their sums through distributed shared memory.
// Tiles of one expert's lines follow each other, so that the clusters at work together read neighbouring memory.
template <int NT, class T>
__global__ void __launch_bounds__(kRowsThreads)
experts_rows_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ ExpertParams p) {
  using S = ExpertRowsShape<NT>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  ExpertRowsShared* sh = reinterpret_cast<ExpertRowsShared*>(tiles + S::kStages * S::kStageBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank(), size = (int)cluster_size();
  const int index = (int)(blockIdx.x / size), n0 = index % p.tiles_n * 128;
  const int g_begin = (int)((int64_t)rank * p.groups / size), g_end = (int)((int64_t)(rank + 1) * p.groups / size);
  const int b_begin = 4 * g_begin, b_end = min(4 * g_end, p.x.blocks);

  if (warp == 0) {
    const RowsTile found = rows_tile(p.offsets, p.experts, p.rows, index / p.tiles_n, NT, lane);
    if (lane == 0) sh->tile = found;
  } else if (warp == 1) {
    tmem_alloc(smem_u32(&sh->tmem_base), S::kCols);
    tmem_relinquish();
  } else if (threadIdx.x == 64) {
    prefetch_tensormap(&map_x);
    prefetch_tensormap(&map_w);
    for (int s = 0; s < 4; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1), mbar_init(smem_u32(&sh->empty[s]), 1);
      mbar_init(smem_u32(&sh->sf_full[s]), 4), mbar_init(smem_u32(&sh->sf_empty[s]), 1);
    }
    mbar_init(smem_u32(&sh->acc_full), 1);
    mbar_init(smem_u32(&sh->drained), 1);
    sh->abort = 0;
    fence_barrier_init();
    fence_proxy_async();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh->tmem_base;
  const RowsTile tile = sh->tile;
  if (p.clear) {
    const int rest = tile.first + p.rows - tile.behind;
    T* out = static_cast<T*>(p.out);
    for (int i = (int)blockIdx.x; i < rest; i += (int)gridDim.x) {
      T* row = out + (int64_t)(i < tile.first ? i : i - tile.first + tile.behind) * p.ldc;
      for (int n = threadIdx.x; n < p.N; n += kRowsThreads) store_element(row + n, 0.f);
    }
  }
  if (tile.count == 0) {   // the whole cluster: there are at most as many tiles as were launched
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, S::kCols);
    return;
  }
  float* sums = reinterpret_cast<float*>(tiles);   // [NT][128] once the operands have been consumed

  if (warp == 0) {
    if (lane == 0) {
      int issued = 0;
      for (int b = b_begin; b < b_end; ++b, ++issued) {
        const int stage = issued % S::kStages;
        if (!wait_bounded(smem_u32(&sh->empty[stage]), ((uint32_t)(issued / S::kStages) & 1u) ^ 1u, &sh->abort, p.status, 0xC00 + stage)) break;
        const uint32_t dst = smem_u32(tiles + stage * S::kStageBytes), full = smem_u32(&sh->full[stage]);
        mbar_arrive_expect_tx(full, S::kStageBytes);
        int x, y;
        tile_at(p.w.contract_rows, n0, b, x, y);
        tma_load_3d(dst, &map_w, full, x, y, tile.expert);
        tma_load_2d(dst + S::kWBytes, &map_x, full, b * kBlock, tile.t0);
      }
      if (sh->abort) {   // copies in flight land before this CTA leaves
        const uint64_t t0 = global_timer_ns();
        for (int j = max(0, issued - S::kStages); j < issued; ++j)
          while (!mbar_try_wait(smem_u32(&sh->full[j % S::kStages]), (uint32_t)(j / S::kStages) & 1u) && global_timer_ns() - t0 < kWaitLimitNs) {
          }
      }
    }
  } else if (warp == 1) {
    const int w_lines = p.w.contract_rows;
    const uint32_t w_step = operand_step(w_lines), x_step = operand_step(0), idesc = idesc_mxf8(128, NT, w_lines, 0);
    for (int b = b_begin; b < b_end; ++b) {
      const int i = b - b_begin, stage = i % S::kStages, set = (i / 4) % S::kSets;
      if (i % 4 == 0 && !wait_warp(smem_u32(&sh->sf_full[set]), (uint32_t)(i / 4 / S::kSets) & 1u, &sh->abort, p.status, 0xC11)) break;
      if (!wait_warp(smem_u32(&sh->full[stage]), (uint32_t)(i / S::kStages) & 1u, &sh->abort, p.status, 0xC20 + stage)) break;
      tc_fence_after();
      const uint32_t base = smem_u32(tiles + stage * S::kStageBytes);
      const uint64_t dw = operand_desc(w_lines, base), dx = operand_desc(0, base + S::kWBytes);
      if (elect_one()) {
#pragma unroll
        for (uint32_t ks = 0; ks < 4; ++ks)
          mma_mxf8(tmem, dw + ks * w_step, dx + ks * x_step, idesc | idesc_mxf8_block((uint32_t)b & 3u), tmem + NT + set * 8, tmem + NT + set * 8 + 4, (i || ks) ? 1u : 0u);
        mma_commit(smem_u32(&sh->empty[stage]));
        if (b + 1 == b_end) mma_commit(smem_u32(&sh->acc_full));
        if (i % 4 == 3 || b + 1 == b_end) mma_commit(smem_u32(&sh->sf_empty[set]));
      }
      __syncwarp();
    }
    if (sh->abort && elect_one()) {
      mma_commit(smem_u32(&sh->drained));
      const uint64_t t0 = global_timer_ns();
      while (!mbar_try_wait(smem_u32(&sh->drained), 0u) && global_timer_ns() - t0 < kWaitLimitNs) {
      }
    }
  } else {
    const uint32_t quad = (uint32_t)(warp & 3);
    const uint32_t lanes = tmem + ((quad * 32u) << 16);
    const int line = (int)quad * 32 + lane;   // of the 128
    bool ok = true;
    Operand w = p.w;
    w.scales = static_cast<const uint8_t*>(p.w.scales) + tile.expert * p.w_scale_step;
    for (int g = g_begin; g < g_end; ++g) {
      const int i = g - g_begin, set = i % S::kSets;
      uint32_t ww[4], wx[4];
      scale_words<4>(w, n0, lane, g, ww);
      scale_words<(NT + 31) / 32>(p.x, tile.t0, lane, g, wx);
      if (!wait_warp(smem_u32(&sh->sf_empty[set]), ((uint32_t)(i / S::kSets) & 1u) ^ 1u, &sh->abort, p.status, 0xC31)) {
        ok = false;
        break;
      }
      tc_fence_after();
      tmem_st_32x4(lanes + NT + set * 8, ww);
      tmem_st_32x4(lanes + NT + set * 8 + 4, wx);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh->sf_full[set]));
    }
    if (ok) ok = wait_warp(smem_u32(&sh->acc_full), 0u, &sh->abort, p.status, 0xC32);
    if (ok) {
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < NT / 16; ++c) {
        uint32_t d[16];
        tmem_ld_32x16(lanes + c * 16, d);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[(c * 16 + e) * 128 + line] = __uint_as_float(d[e]);
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem, S::kCols);
  }
  // each CTA of the cluster joins its share of the sums, in the order of the ranges, four columns a thread
  const uint32_t local = smem_u32(sums);
  for (int e = rank * kRowsThreads + (int)threadIdx.x; e < tile.count * 32; e += size * kRowsThreads) {
    const int n = n0 + e % 32 * 4, left = p.N - n;
    if (left <= 0) continue;
    float4 v[kRowsMostCluster];
#pragma unroll
    for (int r = 0; r < kRowsMostCluster; ++r)
      if (r < size) v[r] = load_cluster_f32x4(map_to_cta(local + (uint32_t)e * 16u, (uint32_t)r));
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < kRowsMostCluster; ++r)
      if (r < size) sum[0] += v[r].x, sum[1] += v[r].y, sum[2] += v[r].z, sum[3] += v[r].w;
    T* c = static_cast<T*>(p.out) + (int64_t)(tile.t0 + e / 32) * p.ldc + n;
    if (sizeof(T) == 2 && p.wide_ok && left >= 4) {
      *reinterpret_cast<uint2*>(c) = make_uint2(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]));
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < left) store_element(c + k, sum[k]);
    }
  }
  asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");   // no CTA leaves while another reads its sums; nothing was written that another waits for
  cluster_wait();
}

// ---- weight gradients -------------------------------------------------------------------
// 256 x 256 tiles; both operands are summed over their rows, expert e's blocks of 128 rows being before[e] .. before[e+1] - 1.
constexpr int kTile = 256;
struct SegmentParams {
  Operand a, b;
  Output out;           // one expert's
  int64_t out_step;     // bytes from one expert's result to the next
  const int* offsets;
  int experts, rows, tiles_m, tiles_n;
  int chunk;            // blocks summed in tensor memory before the sum is added to C in FP32, a multiple of 4
  StatusBlock* status;
};
struct SegmentShape {
  static constexpr int kABytes = 128 * kBlock, kBBytes = 128 * kBlock, kStageBytes = kABytes + kBBytes;
  static constexpr int kBufferStep = 224;   // the accumulators share 32 columns: a new tile waits until those of the previous one have been read
  static constexpr size_t kSmem = (size_t)kPairStages * kStageBytes + kEpilogueWarps * 4096 + 512 + 1024;
};
struct SegmentItem {
  int expert, m0, n0, b_begin, b_end;
};
// Items expert by expert, in bands of rows of tiles.  There is no room for a table of the segments: each warp follows the offsets, which
// never fall and stay within the rows, as it goes.
struct SegmentWalk {
  const SegmentParams& p;
  int expert = 0, end, b_begin = 0, b_end;
  __device__ __forceinline__ explicit SegmentWalk(const SegmentParams& q) : p(q) {
    end = min(max(__ldg(p.offsets), 0), p.rows);
    b_end = 0;
    take();
  }
  __device__ __forceinline__ void take() {
    const int begin = end;
    end = min(max(__ldg(p.offsets + expert + 1), begin), p.rows);
    b_begin = b_end;
    b_end += (end - begin + kBlock - 1) / kBlock;
  }
  __device__ __forceinline__ SegmentItem at(int item) {
    const int tiles = p.tiles_m * p.tiles_n, e = item / tiles, tile = item - e * tiles;
    while (expert < e) ++expert, take();
    const int band = kGroupBand * p.tiles_n, g = tile / band, rem = tile - g * band, rows = min(kGroupBand, p.tiles_m - kGroupBand * g);
    return {e, (kGroupBand * g + rem % rows) * kTile, rem / rows * kTile, b_begin, b_end};
  }
};

template <bool kBf16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
segments_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_c,
                     const __grid_constant__ SegmentParams p) {
  using S = SegmentShape;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* staging = tiles + kPairStages * S::kStageBytes;
  ExpertShared* sh = reinterpret_cast<ExpertShared*>(staging + kEpilogueWarps * 4096);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const int items = p.tiles_m * p.tiles_n * p.experts;
  SegmentWalk walk(p);

  if (threadIdx.x == 0) {
    prefetch_tensormap(&map_a);
    prefetch_tensormap(&map_b);
    prefetch_tensormap(&map_c);
    init_barriers(sh);
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&sh->tmem_base), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem = sh->tmem_base;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int item = pair; item < items && ok; item += npairs) {
        const SegmentItem it = walk.at(item);
        for (int b = it.b_begin; b < it.b_end; ++b) {
          if (!wait_bounded(smem_u32(&sh->empty[stage]), phase ^ 1u, &sh->abort, p.status, 0xB00 + stage)) {
            ok = false;
            break;
          }
          const uint32_t full = map_to_cta(smem_u32(&sh->full[stage]), 0);
          const uint32_t dst = smem_u32(tiles + stage * S::kStageBytes);
          if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh->full[stage]), 2 * S::kStageBytes);
          tma_load_2d_pair(dst, &map_a, full, it.m0 + rank * 128, b * kBlock);
          tma_load_2d_pair(dst + S::kABytes, &map_b, full, it.n0 + rank * 128, b * kBlock);
          ++issued;
          if (++stage == kPairStages) stage = 0, phase ^= 1u;
        }
      }
      if (sh->abort && rank == 0) drain_copies(sh->full, issued);
    }
  } else if (warp == 1) {
    if (rank == 0) {
      int stage = 0;
      uint32_t phase = 0, unit = 0, sf_unit = 0;
      const uint32_t step = operand_step(1), idesc = idesc_mxf8(kTile, kTile, 1, 1);
      bool ok = true;
      for (int item = pair; item < items && ok; item += npairs) {
        const SegmentItem it = walk.at(item);
        if (it.b_begin == it.b_end) continue;
        for (int c0 = it.b_begin & ~3; c0 < it.b_end && ok; c0 += p.chunk, ++unit) {
          const int b_begin = max(it.b_begin, c0), b_end = min(it.b_end, c0 + p.chunk);
          const uint32_t buf = unit & 1u, acc = tmem + buf * S::kBufferStep;
          if (!wait_warp(smem_u32(&sh->acc_empty[buf]), ((unit >> 1) & 1u) ^ 1u, &sh->abort, p.status, 0xB10)) { ok = false; break; }
          if (unit && !wait_warp(smem_u32(&sh->overlap), (unit - 1) & 1u, &sh->abort, p.status, 0xB11)) { ok = false; break; }
          tc_fence_after();
          for (int b = b_begin; b < b_end; ++b) {
            const uint32_t set = sf_unit & 1u, sfa = tmem + kScaleCol + set * 12, sfb = sfa + 4;
            if (((b & 3) == 0 || b == b_begin) && !wait_warp(smem_u32(&sh->sf_full[set]), (sf_unit >> 1) & 1u, &sh->abort, p.status, 0xB13)) { ok = false; break; }
            if (!wait_warp(smem_u32(&sh->full[stage]), phase, &sh->abort, p.status, 0xB20 + stage)) { ok = false; break; }
            tc_fence_after();
            const uint32_t base = smem_u32(tiles + stage * S::kStageBytes);
            const uint64_t da = operand_desc(1, base), db = operand_desc(1, base + S::kABytes);
            const bool last = b + 1 == b_end, last_of_scales = (b & 3) == 3 || last;
            if (elect_one()) {
#pragma unroll
              for (uint32_t ks = 0; ks < 4; ++ks)
                mma_mxf8_pair(acc, da + ks * step, db + ks * step, idesc | idesc_mxf8_block((uint32_t)b & 3u), sfa, sfb, (b > b_begin || ks) ? 1u : 0u);
              mma_commit_pair(smem_u32(&sh->empty[stage]), (uint16_t)3);
              if (last_of_scales) mma_commit_pair(smem_u32(&sh->sf_empty[set]), (uint16_t)3);
              if (last) mma_commit_pair(smem_u32(&sh->acc_full[buf]), (uint16_t)3);
            }
            __syncwarp();
            if (++stage == kPairStages) stage = 0, phase ^= 1u;
            sf_unit += last_of_scales;
          }
        }
      }
      if (sh->abort && elect_one()) drain_products(&sh->drained);
    }
  } else if (warp < kFirstEpilogue) {
    // The words of a group of four blocks serve two experts where a segment ends inside it: each takes its own bytes of them.
    const uint32_t at = tmem + (((uint32_t)(warp & 3) * 32u) << 16) + kScaleCol;
    const uint32_t leader = map_to_cta(smem_u32(&sh->sf_full[0]), 0);
    uint32_t unit = 0;
    bool ok = true;
    for (int item = pair; item < items && ok; item += npairs) {
      const SegmentItem it = walk.at(item);
      if (it.b_begin == it.b_end) continue;
      const int g_begin = it.b_begin / 4, g_end = (it.b_end + 3) / 4;
      uint32_t wa[4], wb0[4], wb1[4];
      auto fetch = [&](int g) {
        scale_words<4>(p.a, it.m0 + rank * 128, lane, g, wa);
        scale_words<4>(p.b, it.n0, lane, g, wb0);
        scale_words<4>(p.b, it.n0 + 128, lane, g, wb1);
      };
      fetch(g_begin);
      for (int g = g_begin; g < g_end; ++g, ++unit) {
        const uint32_t set = unit & 1u;
        if (!wait_warp(smem_u32(&sh->sf_empty[set]), ((unit >> 1) & 1u) ^ 1u, &sh->abort, p.status, 0xB30)) {
          ok = false;
          break;
        }
        tc_fence_after();
        tmem_st_32x4(at + set * 12, wa);
        tmem_st_32x4(at + set * 12 + 4, wb0);
        tmem_st_32x4(at + set * 12 + 8, wb1);
        if (g + 1 < g_end) fetch(g + 1);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(leader + set * 8);
      }
    }
  } else {
    const uint32_t quad = (uint32_t)(warp & 3);
    const int part = (warp - kFirstEpilogue) >> 2;   // which 128 of the columns
    uint8_t* box = staging + (warp - kFirstEpilogue) * 4096;
    const uint32_t lanes = tmem + ((quad * 32u) << 16);
    const uint32_t empty0 = map_to_cta(smem_u32(&sh->acc_empty[0]), 0), overlap = map_to_cta(smem_u32(&sh->overlap), 0);
    constexpr int kPieces = kBf16 ? 2 : 4, kWidth = kBf16 ? 64 : 32;
    uint32_t unit = 0;
    bool ok = true;
    for (int item = pair; item < items && ok; item += npairs) {
      const SegmentItem it = walk.at(item);
      const int m = it.m0 + rank * 128 + (int)quad * 32, n = it.n0 + part * 128;
      Output out = p.out;
      out.ptr = static_cast<uint8_t*>(p.out.ptr) + it.expert * p.out_step;
      if (it.b_begin == it.b_end) {   // an expert without rows: its sum is empty
        const uint32_t w[32] = {};
        for (int c = 0; c < kPieces && !out.add; ++c) store_box<kBf16>(out, &map_c, box, lane, w, m, n + c * kWidth, it.expert, false);
        continue;
      }
      for (int c0 = it.b_begin & ~3; c0 < it.b_end; c0 += p.chunk, ++unit) {
        const uint32_t buf = unit & 1u;
        const bool later = c0 > it.b_begin;   // a later range of the same tile is added to the earlier ones
        if (later && p.out.tma && lane == 0) bulk_wait();
        if (!wait_warp(smem_u32(&sh->acc_full[buf]), (unit >> 1) & 1u, &sh->abort, p.status, 0xB41)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t from = lanes + buf * S::kBufferStep + part * 128;
        const bool shared_half = buf == 0 ? part == 1 : part == 0;   // holds the columns that the other accumulator shares
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int c = buf == 0 && part == 1 ? kPieces - 1 - i : i;   // those columns first
          uint32_t w[32];
          if constexpr (kBf16) {
            uint32_t d0[32], d1[32];
            tmem_ld_32x32(from + c * 64, d0);
            tmem_ld_32x32(from + c * 64 + 32, d1);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              w[e] = pack_bf16(__uint_as_float(d0[2 * e]), __uint_as_float(d0[2 * e + 1]));
              w[16 + e] = pack_bf16(__uint_as_float(d1[2 * e]), __uint_as_float(d1[2 * e + 1]));
            }
          } else {
            tmem_ld_32x32(from + c * 32, w);
            tmem_wait_ld();
          }
          if ((i == 0 && shared_half) || i == kPieces - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              if (i == 0 && shared_half) mbar_arrive_cluster(overlap);
              if (i == kPieces - 1) mbar_arrive_cluster(empty0 + buf * 8);
            }
          }
          store_box<kBf16>(out, &map_c, box, lane, w, m, n + c * kWidth, it.expert, out.add || later);
        }
      }
    }
    if (lane == 0) bulk_wait();   // the staging memory is read until then
  }

  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc_pair(tmem, 512);
  }
}

// Rows that belong to a segment (an empty sum), or those that do not, become zero: results of products over nothing.
template <class T>
__global__ void __launch_bounds__(256) clear_rows_kernel(const int* offsets, int experts, int rows, T* out, int64_t ldc, int N, int rest_too) {
  const int begin = min(max(offsets[0], 0), rows);
  int end = begin;   // the largest offset within the rows: segments lie side by side up to it
  for (int e = threadIdx.x; e < experts; e += 256) end = max(end, min(offsets[e + 1], rows));
  end = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)end);
  __shared__ int ends[8];
  if (threadIdx.x % 32 == 0) ends[threadIdx.x / 32] = end;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) end = max(end, ends[i]);
  for (int r = blockIdx.x; r < rows; r += gridDim.x) {
    if (!rest_too && (r < begin || r >= end)) continue;
    for (int n = threadIdx.x; n < N; n += 256) out[(int64_t)r * ldc + n] = T(0);
  }
}

// ---- host side ------------------------------------------------------------------------
bool expert_map(CUtensorMap* map, const ozk_fp8_experts& w, int64_t experts, int64_t rows, int64_t cols) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)experts};
  const cuuint64_t strides[2] = {(cuuint64_t)w.ld, (cuuint64_t)w.stride};
  const cuuint32_t box[3] = {(cuuint32_t)kBlock, (cuuint32_t)kBlock, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<uint8_t*>(w.codes), dims, strides, box, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

template <bool kBf16>
bool launch_experts_pair(const ExpertMaps& maps, const ExpertParams& p, int pairs, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto kernel = experts_pair_kernel<kBf16>;
  if (!raise_smem(kernel, ExpertShape::smem(kMostExperts), done)) return false;
  kernel<<<(unsigned)(2 * pairs), kPairThreads, ExpertShape::smem(p.experts), st>>>(maps, p);
  return cudaGetLastError() == cudaSuccess;
}
template <bool kBf16>
bool launch_segments_pair(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, const SegmentParams& p, int pairs, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto kernel = segments_pair_kernel<kBf16>;
  if (!raise_smem(kernel, SegmentShape::kSmem, done)) return false;
  kernel<<<(unsigned)(2 * pairs), kPairThreads, SegmentShape::kSmem, st>>>(a, b, c, p);
  return cudaGetLastError() == cudaSuccess;
}

template <int NT, class T>
bool launch_experts_rows(const ExpertMaps& maps, const ExpertParams& p, int64_t tiles, int cluster, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto kernel = experts_rows_kernel<NT, T>;
  if (!raise_smem(kernel, ExpertRowsShape<NT>::kSmem, done)) return false;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * cluster), 1, 1);
  cfg.blockDim = dim3(kRowsThreads, 1, 1);
  cfg.dynamicSmemBytes = ExpertRowsShape<NT>::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, maps.x[0], maps.w, p) == cudaSuccess;
}
template <class T>
bool launch_experts_rows(int nt, const ExpertMaps& maps, const ExpertParams& p, int64_t tiles, int cluster, cudaStream_t st) {
  return nt == 16 ? launch_experts_rows<16, T>(maps, p, tiles, cluster, st) : nt == 32 ? launch_experts_rows<32, T>(maps, p, tiles, cluster, st) : launch_experts_rows<64, T>(maps, p, tiles, cluster, st);
}

// Tiles of at most `height` rows that any segments of these rows need.
int64_t most_tiles(int64_t rows, int64_t experts, int height) { return (rows + (height - 1) * (experts < rows ? experts : rows)) / height; }

// How experts_rows_kernel would run: NT rows a tile (0: it does not), `cluster` CTAs along K.  The host knows the mean of the rows of an expert, not how they lie.
// It serves up to 8 rows an expert, and up to 64 where the pairs have too few tiles to be at work all.  Rows against pairs, us: 244 rows of 32 experts (4096 -> 2048) 46.6 : 51.9,
// 64 of 8 (4096 -> 4096) 26.5 : 30.0, 8 of 64 (2048 -> 4096) 18.0 : 21.1, but 1000 of 64 (2048 -> 2048) 57.8 : 52.0.  Between 8 and 16 rows an expert, nearly even ones, rows
// against pairs: 320 of 32 (4096 -> 2048) 51.7 : 54.7, 160 of 16 (4096 -> 4096) 51.4 : 53.9, but 640 of 64 (2048 -> 4096) 106.8 : 95.4, 1280 of 128 (2048 -> 1024) 59.9 : 56.2: what
// decides there is how many experts there are as much as their rows, within 12 % either way, so the limit stays at 8.
// K is split only while CTAs are missing: 64 of 8 26.5, split by two 30.0; one row (4096 -> 4096) 14.9, split by eight 10.7.
struct ExpertRowsPlan {
  int nt, cluster;
  int64_t tiles;
};
ExpertRowsPlan expert_rows_plan(int64_t rows, int64_t experts, int64_t N, int groups, bool bf16, int sms) {
  ExpertRowsPlan r = {};
  const int64_t used = experts < rows ? experts : rows;
  if (rows > 8 * used && (rows > 64 * used || most_tiles(rows, experts, kTokens) * ceil_div(N, kLines) >= sms / 2)) return r;
  r.nt = rows <= 4 * used ? 16 : rows <= 16 * used ? 32 : 64;
  r.tiles = most_tiles(rows, experts, r.nt) * ceil_div(N, 128);
  int64_t c = r.tiles >= 2 * sms ? 1 : 2 * sms / r.tiles;   // two CTAs fit a multiprocessor: K is split over a cluster while that fills them
  if (!bf16 && c * kRowsRange < groups) c = ceil_div(groups, kRowsRange);   // FP32 results: short ranges
  if (c > groups) c = groups;
  if (c > kRowsMostCluster) c = kRowsMostCluster;
  r.cluster = (int)c;
  if (!bf16 && c * kRowsRange < groups) r.nt = 0;
  return r;
}

constexpr int64_t kMostRows = INT32_MAX - 65536;   // rows are cleared in steps of 8 a multiprocessor, whose last one passes them
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// Codes that a tensor map may be made of.
bool good_operand(const uint8_t* codes, int64_t ld, const void* scales, int64_t cols, uintptr_t scale_align) {
  return codes && scales && aligned(codes, 16) && ld % 16 == 0 && ld >= cols && aligned(scales, scale_align);
}

}  // namespace
}  // namespace ozk

using namespace ozk;

extern "C" {

int64_t ozk_fp8_segment_blocks(int64_t rows, int64_t experts) {
  if (rows < 0 || experts < 0) return 0;
  return (rows + 127 * (experts < rows ? experts : rows)) / 128;
}

ozk_status ozk_fp8_grouped_gemm(int64_t rows, int64_t N, int64_t K, const ozk_fp8_operand* X, const ozk_fp8_experts* W, int64_t experts, const int32_t* offsets,
                                void* C, int c_type, int64_t ldc, int clear_rest, void* status, void* stream) {
  if (rows < 0 || N < 0 || K < 0 || experts < 0 || !X || !W || (c_type != OZK_F32 && c_type != OZK_BF16) || ldc < N) return OZK_ERR_INVALID_ARG;
  if ((clear_rest != 0 && clear_rest != 1) || (W->contract_rows != 0 && W->contract_rows != 1)) return OZK_ERR_INVALID_ARG;
  const int64_t most = INT32_MAX - 1024;
  if (rows > kMostRows || N > most || K > most || experts > kMostExperts) return OZK_ERR_UNSUPPORTED;
  if (rows == 0 || N == 0) return OZK_OK;
  const bool bf16 = c_type == OZK_BF16;
  const size_t size = bf16 ? 2 : 4;
  if (!C || !aligned(C, size)) return OZK_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (experts == 0) {
    if (clear_rest && cudaMemset2DAsync(C, (size_t)ldc * size, 0, (size_t)N * size, (size_t)rows, st) != cudaSuccess) return OZK_ERR_CUDA;
    return OZK_OK;
  }
  if (!offsets || !aligned(offsets, 4)) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  const int sms = device_sm_count();
  if (sms < 2) return OZK_ERR_CUDA;
  if (K == 0) {
    const unsigned grid = (unsigned)(rows < 8 * sms ? rows : 8 * sms);
    if (bf16) clear_rows_kernel<uint16_t><<<grid, 256, 0, st>>>(offsets, (int)experts, (int)rows, static_cast<uint16_t*>(C), ldc, (int)N, clear_rest);
    else clear_rows_kernel<float><<<grid, 256, 0, st>>>(offsets, (int)experts, (int)rows, static_cast<float*>(C), ldc, (int)N, clear_rest);
    return cudaGetLastError() == cudaSuccess ? OZK_OK : OZK_ERR_CUDA;
  }
  const int64_t w_rows = W->contract_rows ? K : N, w_cols = W->contract_rows ? N : K;
  if (X->contract_rows != 0 || X->scale_kind != OZK_SCALE_LINES) return OZK_ERR_UNSUPPORTED;
  if (!good_operand(X->codes, X->ld, X->scales, K, 4) || !good_operand(W->codes, W->ld, W->scales, w_cols, 1)) return OZK_ERR_INVALID_ARG;
  if (W->stride % 16 || (experts > 1 && W->stride < (w_rows - 1) * W->ld + w_cols)) return OZK_ERR_INVALID_ARG;
  if (!status) return OZK_ERR_WORKSPACE;
  if (!aligned(status, 256)) return OZK_ERR_INVALID_ARG;

  ExpertParams p = {};
  p.x = Operand{X->codes, X->ld, X->scales, OZK_SCALE_LINES, 0, (int)rows, (int)ceil_div(K, kBlock), 0};
  p.w = Operand{W->codes, W->ld, W->scales, OZK_SCALE_TILES, W->contract_rows, (int)N, (int)ceil_div(K, kBlock), ceil_div(w_cols, kBlock)};
  p.w_scale_step = ceil_div(w_rows, kBlock) * ceil_div(w_cols, kBlock);
  p.offsets = offsets;
  p.experts = (int)experts, p.rows = (int)rows;
  p.out = C, p.ldc = ldc, p.N = (int)N, p.tiles_n = (int)ceil_div(N, kLines), p.groups = (int)ceil_div(K, kGroupK);
  p.chunk = bf16 ? 4 * p.groups : 4 * kRangeGroups;
  p.pairs_ok = aligned(C, 4) && ldc % 2 == 0, p.wide_ok = aligned(C, 8) && ldc % 4 == 0, p.pieces_ok = aligned(C, 16) && ldc % 8 == 0;
  p.clear = clear_rest;
  p.status = static_cast<StatusBlock*>(status);
  const ExpertRowsPlan few = expert_rows_plan(rows, experts, N, p.groups, bf16, sms);
  const int64_t tiles = most_tiles(rows, experts, kTokens);
  if ((tiles * p.tiles_n + sms) * ceil_div(p.groups, kRangeGroups) > INT32_MAX) return OZK_ERR_UNSUPPORTED;
  ozk_fp8_experts w = *W;
  if (w.stride == 0) w.stride = w.ld * w_rows;   // a single expert's is not used, but a map wants one
  ExpertMaps maps;
  if (!expert_map(&maps.w, w, experts, w_rows, w_cols)) return OZK_ERR_CUDA;
  if (few.nt) {
    if (few.tiles * few.cluster > INT32_MAX) return OZK_ERR_UNSUPPORTED;
    if (!operand_map(&maps.x[0], p.x, K, few.nt)) return OZK_ERR_CUDA;
    p.tiles_n = (int)ceil_div(N, 128);
    return (bf16 ? launch_experts_rows<__nv_bfloat16>(few.nt, maps, p, few.tiles, few.cluster, st) : launch_experts_rows<float>(few.nt, maps, p, few.tiles, few.cluster, st)) ? OZK_OK : OZK_ERR_CUDA;
  }
  for (int i = 0; i < kXBoxes; ++i)
    if (!operand_map(&maps.x[i], p.x, K, x_box(i))) return OZK_ERR_CUDA;
  const int64_t items = tiles * p.tiles_n;
  const int pairs = (int)(items < sms / 2 ? items : sms / 2);
  return (bf16 ? launch_experts_pair<true>(maps, p, pairs, st) : launch_experts_pair<false>(maps, p, pairs, st)) ? OZK_OK : OZK_ERR_CUDA;
}

ozk_status ozk_fp8_segment_gemm(int64_t experts, int64_t M, int64_t N, int64_t rows, const ozk_fp8_operand* A, const ozk_fp8_operand* B, const int32_t* offsets,
                                void* C, int c_type, int64_t ldc, int64_t stride, int accumulate, void* status, void* stream) {
  if (experts < 0 || M < 0 || N < 0 || rows < 0 || !A || !B || (c_type != OZK_F32 && c_type != OZK_BF16) || ldc < N) return OZK_ERR_INVALID_ARG;
  if ((accumulate != 0 && accumulate != 1) || (experts > 1 && stride < (M - 1) * ldc + N)) return OZK_ERR_INVALID_ARG;
  const int64_t most = INT32_MAX - 1024;
  const int64_t blocks = ozk_fp8_segment_blocks(rows, experts);   // up to 127 rows an expert more than there are, and indexed by ints too
  if (rows > most || blocks * kBlock > INT32_MAX || M > most || N > most || experts > kMostExperts || (accumulate && c_type != OZK_F32)) return OZK_ERR_UNSUPPORTED;
  if (experts == 0 || M == 0 || N == 0) return OZK_OK;
  const bool bf16 = c_type == OZK_BF16;
  const size_t size = bf16 ? 2 : 4;
  if (!C || !aligned(C, size)) return OZK_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (accumulate) return OZK_OK;
    for (int64_t e = 0; e < experts; ++e)
      if (cudaMemset2DAsync(static_cast<uint8_t*>(C) + e * stride * size, (size_t)ldc * size, 0, (size_t)N * size, (size_t)M, st) != cudaSuccess) return OZK_ERR_CUDA;
    return OZK_OK;
  }
  if (!offsets || !aligned(offsets, 4)) return OZK_ERR_INVALID_ARG;
  if (A->contract_rows != 1 || B->contract_rows != 1 || A->scale_kind != OZK_SCALE_LINES || B->scale_kind != OZK_SCALE_LINES) return OZK_ERR_UNSUPPORTED;
  if (!good_operand(A->codes, A->ld, A->scales, M, 4) || !good_operand(B->codes, B->ld, B->scales, N, 4)) return OZK_ERR_INVALID_ARG;
  if (!status) return OZK_ERR_WORKSPACE;
  if (!aligned(status, 256)) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  const int sms = device_sm_count();
  if (sms < 2) return OZK_ERR_CUDA;

  SegmentParams p = {};
  p.a = Operand{A->codes, A->ld, A->scales, OZK_SCALE_LINES, 1, (int)M, (int)blocks, 0};
  p.b = Operand{B->codes, B->ld, B->scales, OZK_SCALE_LINES, 1, (int)N, (int)blocks, 0};
  const bool tma = aligned(C, 16) && ((size_t)ldc * size) % 16 == 0 && (experts == 1 || ((size_t)stride * size) % 16 == 0);
  p.out = Output{C, ldc, (int)M, (int)N, accumulate, tma ? 1 : 0};
  p.out_step = stride * (int64_t)size;
  p.offsets = offsets;
  p.experts = (int)experts, p.rows = (int)rows;
  p.tiles_m = (int)ceil_div(M, kTile), p.tiles_n = (int)ceil_div(N, kTile);
  p.chunk = bf16 ? (int)round_up(blocks, 4) + 4 : 4 * kRangeGroups;
  p.status = static_cast<StatusBlock*>(status);
  const int64_t items = experts * ceil_div(M, kTile) * ceil_div(N, kTile);
  if (items + sms > INT32_MAX) return OZK_ERR_UNSUPPORTED;
  CUtensorMap map_a, map_b, map_c;
  if (!operand_map(&map_a, p.a, blocks * kBlock, 128) || !operand_map(&map_b, p.b, blocks * kBlock, 128)) return OZK_ERR_CUDA;
  if (tma) {
    const cuuint64_t dims[3] = {(cuuint64_t)N, (cuuint64_t)M, (cuuint64_t)experts};
    const cuuint64_t strides[2] = {(cuuint64_t)ldc * size, (cuuint64_t)(experts == 1 ? ldc * M : stride) * size};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / size), 32, 1};
    if (!encode(&map_c, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, C, dims, strides, box, CU_TENSOR_MAP_L2_PROMOTION_NONE)) return OZK_ERR_CUDA;
  } else {
    map_c = map_a;   // not used
  }
  const int pairs = (int)(items < sms / 2 ? items : sms / 2);
  return (bf16 ? launch_segments_pair<true>(map_a, map_b, map_c, p, pairs, st) : launch_segments_pair<false>(map_a, map_b, map_c, p, pairs, st)) ? OZK_OK : OZK_ERR_CUDA;
}

}  // extern "C"
