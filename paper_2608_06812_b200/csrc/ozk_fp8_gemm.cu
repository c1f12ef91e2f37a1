// The block-scaled product C[m,n] = sum_k A(m,k) sa(m,k/128) B(n,k) sb(n,k/128) of E4M3 operands on the tensor cores.
//
// UE8M0 scales: tcgen05.mma kind::mxf8f6f4 takes a scale byte for each operand row and 32 values of k.  Four
//   instructions of one block of 128 are given the same byte, so that a 32-bit word of scale bytes per row serves
//   512 values of k, and the product needs no arithmetic besides the tensor cores'.
// FP32 scales: kind::f8f6f4 sums each block of 128 by itself; the epilogue warps multiply it by its scales and add it up
//   in registers while the tensor cores form the next blocks.
//
// An operand whose k runs along its rows (contract_rows) is not transposed: its tiles are fetched with the 128-byte
// rows along the lines, and the instruction reads them that way.
//
// Two kernels.  product_pair_kernel: a pair of CTAs forms 256 x 256 tiles of C one after another, with the TMA producer, the MMA
//   issuer, the scale writers and the epilogue in warps of their own; where there are few tiles K is split over several pairs and
//   join_kernel adds the partial sums in order.  Bound by the tensor cores and, back to back, by the power limit: 8192^3 in 443 us
//   (2.48 PFLOP/s) in a loop of them, 374 us (2.94) in short bursts; the issuer alone, without loads, would take 96 % of the latter's clocks.
//   With FP32 scales the epilogue's reads and multiply-adds hold up the hand-over of the two accumulators: 4096^3 in 79 us
//   (1.75 PFLOP/s), of which 64 us remain without any read or multiply-add.
// product_rows_kernel: few rows of C, where reading B is what costs.  B's lines become the 128 rows of the instruction and up to 128 rows of
//   C its columns; the CTAs of a cluster share a tile's K and add their sums through distributed shared memory, so that one launch does
//   all.  Bound by memory from about 64 MB of B on (1 x 8192 x 8192: 14.8 us, 4.5 TB/s), by launch, set-up and the cluster's barriers below
//   (1 x 4096 x 4096: 7.0 us, of which 0.9 us stream B).
#include <cuda.h>

#include <atomic>

#include "ozk_fp8.cuh"
#include "ozk_ptx.cuh"
#include "ozk_wait.cuh"

namespace ozk {
namespace {

using namespace fp8;
using namespace ptx;

// ---- operands -------------------------------------------------------------------------
struct Operand {
  const uint8_t* codes;
  int64_t ld;
  const void* scales;
  int kind, contract_rows;
  int lines, blocks;   // blocks = ceil(K / 128)
  int64_t tiles;       // tiles (TILES) or blocks per stored row of scales
};

// Scale bytes of blocks 4 g .. 4 g + 3 for the lines line0 + 32 c + lane of 128, c = 0 .. columns - 1; 1 (127) where there is none.
// line0 is a multiple of 128: with TILES all 128 lines have the same word.
template <int kColumns>
__device__ __forceinline__ void scale_words(const Operand& o, int line0, int lane, int g, uint32_t (&w)[4]) {
  if (o.kind == OZK_SCALE_LINES) {
    const uint32_t* s = static_cast<const uint32_t*>(o.scales) + (int64_t)g * o.lines + line0 + lane;
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = c < kColumns && line0 + c * 32 + lane < o.lines ? __ldg(s + c * 32) : 0x7F7F7F7Fu;
  } else {
    const uint8_t* s = static_cast<const uint8_t*>(o.scales);
    const int64_t tile = line0 / kBlock, b0 = 4 * (int64_t)g;
    const int64_t at = o.contract_rows ? b0 * o.tiles + tile : tile * o.tiles + b0, step = o.contract_rows ? o.tiles : 1;
    uint32_t v = 0x7F7F7F7Fu;
    if (line0 < o.lines) {
      v = 0;
#pragma unroll
      for (int b = 0; b < 4; ++b) v |= (uint32_t)(4 * g + b < o.blocks ? __ldg(s + at + b * step) : 127u) << (8 * b);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = v;
  }
}
// Line and block of an FP32-scaled operand.
__device__ __forceinline__ float scale_line_f32(const Operand& o, int line, int b) {
  return line < o.lines ? __ldg(static_cast<const float*>(o.scales) + (int64_t)line * o.tiles + b) : 0.f;
}
__device__ __forceinline__ float scale_tile_f32(const Operand& o, int line, int b) {
  return line < o.lines ? __ldg(static_cast<const float*>(o.scales) + (int64_t)(line / kBlock) * o.tiles + b) : 0.f;
}

// Coordinates of the tile of an operand that starts at `line` and block `b`: its 128-byte rows run along k, or along the lines.
__device__ __forceinline__ void tile_at(int contract_rows, int line, int b, int& x, int& y) {
  x = contract_rows ? line : b * kBlock;
  y = contract_rows ? b * kBlock : line;
}
__device__ __forceinline__ uint64_t operand_desc(int contract_rows, uint32_t addr) {
  return contract_rows ? smem_desc_sw128_lines(addr) : smem_desc_sw128(addr);
}
// Descriptor units (16 bytes) from one instruction's 32 values of k to the next.
__device__ __forceinline__ uint32_t operand_step(int contract_rows) { return contract_rows ? 4096u >> 4 : 32u >> 4; }

struct Output {
  void* ptr;
  int64_t ld;
  int M, N;
  int add;   // add to what is there (FP32)
  int tma;   // 16-byte aligned rows: boxes by TMA
};

struct ProductParams {
  Operand a, b;
  Output out;          // C, or the partial sums [splits][M][ld] when splits > 1
  int tiles_m, tiles_n, splits, groups;   // groups = ceil(K / 512)
  int chunk_groups;    // groups summed in tensor memory before the sum is added to C in FP32
  StatusBlock* status;
};

constexpr int kGroupK = 4 * kBlock;
constexpr int kRangeGroups = 8192 / kGroupK;   // FP32 results: longest range summed by the tensor cores alone
constexpr int kRowsRangeGroups = 8;            // the same in product_rows_kernel, where a shorter one is only a larger cluster

// ---- CTA-pair kernel --------------------------------------------------------------------
constexpr int kTileM = 256;
constexpr int kTileN = 256;
constexpr int kBand = 16;
constexpr int kMaxPairStages = 6;
template <bool kFloat>
struct PairShape {
  // producer, issuer, then 4 scale warps (UE8M0) or 2 idle ones (FP32 scales), and 8 epilogue warps of 32 rows x 128 columns
  static constexpr int kFirstEpilogue = kFloat ? 4 : 6;
  static constexpr int kEpilogueWarps = 8;
  static constexpr int kThreads = 32 * (kFirstEpilogue + kEpilogueWarps);
  // FP32 scales: an epilogue thread keeps its 128 sums in registers.  384 threads are launched with 168 each (64512); the
  // first four warps keep 56 of them, so that the eight of the epilogue may have 224 (7168 + 57344).
  [[maybe_unused]] static constexpr int kLaunchRegs = 168, kFewRegs = 56, kEpilogueRegs = 224;
  static constexpr int kABytes = 128 * kBlock;             // this CTA's 128 lines of A
  static constexpr int kBBytes = kTileN / 2 * kBlock;      // and half of the lines of B
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = 6;
  // Two accumulators in tensor memory.  FP32 scales: one block of 128 each.  UE8M0: they overlap in 32 columns (224..255), so that both
  // and the scale words fit 512: a new tile waits only until those 32 columns of the previous one have been read.
  static constexpr int kBuffers = 2;
  static constexpr int kBufferStep = kFloat ? 256 : 224;
  [[maybe_unused]] static constexpr int kScaleCol = 480;   // two sets of 4 columns for A, 8 for B
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + kEpilogueWarps * 4096 + 512 + 1024;
};
struct __align__(8) PairShared {
  uint64_t full[kMaxPairStages], empty[kMaxPairStages];
  uint64_t sf_full[2], sf_empty[2];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t overlap, drained;
  uint32_t tmem_base;
  volatile int abort;
};
static_assert(sizeof(PairShared) <= 512, "room reserved behind the stages");

struct Item {
  int m0, n0, split, g_begin, g_end;
};
__device__ __forceinline__ Item pair_item(const ProductParams& p, int item) {
  // Bands of kBand row tiles sweep the column tiles, so that the pairs at work at one time share few panels of A and B and each
  // panel of B is read from memory once a band.  8192^3, back to back: 455 us with bands of 8, 443 with 16, 454 with 24, 485 with 32.
  Item r;
  const int tile = item / p.splits;
  r.split = item - tile * p.splits;
  const int band = kBand * p.tiles_n, g = tile / band, rem = tile - g * band;
  const int rows = min(kBand, p.tiles_m - kBand * g);
  r.n0 = rem / rows * kTileN;
  r.m0 = (kBand * g + rem % rows) * kTileM;
  r.g_begin = (int)((int64_t)r.split * p.groups / p.splits);
  r.g_end = (int)((int64_t)(r.split + 1) * p.groups / p.splits);
  return r;
}

// One warp's 32 rows x 128 bytes of results (32 FP32 or 64 BF16 columns; word w of lane r is bytes 4 w .. of row r)
// through 4 KiB of staging.  Rows of the staging box are swizzled as the tensor map says: 16-byte piece j of row r at j ^ (r % 8).
template <bool kBf16>
__device__ __forceinline__ void store_box(const Output& o, const CUtensorMap* map, uint8_t* staging, int lane, const uint32_t (&w)[32], int m, int n, int z,
                                          bool add) {
  if (m >= o.M || n >= o.N) return;   // the same for all lanes
  // A tiled store writes whole 16-byte pieces, also past the map's last column: a box across an edge within such a piece is stored singly.
  constexpr int kWidth = kBf16 ? 64 : 32, kPiece = kBf16 ? 8 : 4;
  const bool tma = o.tma && (n + kWidth <= o.N || o.N % kPiece == 0);
  if (o.tma) {   // an earlier box may still be read from the staging
    if (lane == 0) bulk_wait_read();
    __syncwarp();
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    *reinterpret_cast<uint4*>(staging + lane * 128 + ((j ^ (lane & 7)) * 16)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  if (tma) {
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
      if (!kBf16 && add) tma_add_3d(map, smem_u32(staging), n, m, z); else tma_store_3d(map, smem_u32(staging), n, m, z);
      bulk_commit();
    }
    return;
  }
  __syncwarp();
  const int rows = min(32, o.M - m);
  for (int r = 0; r < rows; ++r) {   // a row at a time: consecutive lanes, consecutive elements
    const uint32_t v = *reinterpret_cast<const uint32_t*>(staging + r * 128 + (((lane / 4) ^ (r & 7)) * 16) + (lane % 4) * 4);
    const int64_t at = (int64_t)(m + r) * o.ld;
    if constexpr (kBf16) {
      uint16_t* c = static_cast<uint16_t*>(o.ptr) + at;
      if (n + 2 * lane < o.N) c[n + 2 * lane] = (uint16_t)v;
      if (n + 2 * lane + 1 < o.N) c[n + 2 * lane + 1] = (uint16_t)(v >> 16);
    } else if (n + lane < o.N) {
      float* c = static_cast<float*>(o.ptr) + at + n + lane;
      *c = add ? *c + __uint_as_float(v) : __uint_as_float(v);
    }
  }
  __syncwarp();
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <bool kFloat, bool kBf16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairShape<kFloat>::kThreads, 1)
product_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_c,
                    const __grid_constant__ ProductParams p) {
  using S = PairShape<kFloat>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* staging = tiles + S::kStages * S::kStageBytes;
  PairShared* sh = reinterpret_cast<PairShared*>(staging + S::kEpilogueWarps * 4096);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const int items = p.tiles_m * p.tiles_n * p.splits;

  if (threadIdx.x == 0) {
    prefetch_tensormap(&map_a);
    prefetch_tensormap(&map_b);
    prefetch_tensormap(&map_c);
    for (int s = 0; s < S::kStages; ++s) mbar_init(smem_u32(&sh->full[s]), 1), mbar_init(smem_u32(&sh->empty[s]), 1);   // full: the leader's only
    for (int s = 0; s < 2; ++s) mbar_init(smem_u32(&sh->sf_full[s]), 8), mbar_init(smem_u32(&sh->sf_empty[s]), 1);      // 4 scale warps of each CTA
    for (int s = 0; s < 2; ++s) mbar_init(smem_u32(&sh->acc_full[s]), 1), mbar_init(smem_u32(&sh->acc_empty[s]), 2 * S::kEpilogueWarps);   // of both CTAs
    mbar_init(smem_u32(&sh->overlap), 8);
    mbar_init(smem_u32(&sh->drained), 1);
    sh->abort = 0;
    fence_barrier_init();
    fence_proxy_async();
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&sh->tmem_base), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();   // the peer's barriers are initialised before anything is sent to them
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem = sh->tmem_base;

  if (warp < S::kFirstEpilogue) {
    if constexpr (kFloat) set_registers_fewer<S::kFewRegs>();
    if (warp == 0) {
      // ------------------------------ TMA producer (both CTAs) ------------------------------
      if (lane == 0) {
        int stage = 0, issued = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int item = pair; item < items && ok; item += npairs) {
          const Item it = pair_item(p, item);
          const int b_end = min(4 * it.g_end, p.a.blocks);
          for (int b = 4 * it.g_begin; b < b_end; ++b) {
            if (!wait_bounded(smem_u32(&sh->empty[stage]), phase ^ 1u, &sh->abort, p.status, 0x800 + stage)) {
              ok = false;
              break;
            }
            const uint32_t full = map_to_cta(smem_u32(&sh->full[stage]), 0);
            const uint32_t dst = smem_u32(tiles + stage * S::kStageBytes);
            if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh->full[stage]), 2 * S::kStageBytes);
            int x, y;
            tile_at(p.a.contract_rows, it.m0 + rank * 128, b, x, y);
            tma_load_2d_pair(dst, &map_a, full, x, y);
            tile_at(p.b.contract_rows, it.n0 + rank * (kTileN / 2), b, x, y);
            tma_load_2d_pair(dst + S::kABytes, &map_b, full, x, y);
            ++issued;
            if (++stage == S::kStages) stage = 0, phase ^= 1u;
          }
        }
        if (sh->abort && rank == 0) {   // copies in flight land before this CTA leaves
          const uint64_t t0 = global_timer_ns();
          for (int j = max(0, issued - S::kStages); j < issued; ++j)
            while (!mbar_try_wait(smem_u32(&sh->full[j % S::kStages]), (uint32_t)(j / S::kStages) & 1u) && global_timer_ns() - t0 < kWaitLimitNs) {
            }
        }
      }
    } else if (warp == 1) {
      // ------------------------------ MMA issuer (leader only) ------------------------------
      // The whole warp walks the loop and waits; one elected lane issues.  Descriptors stay uniform that way.
      if (rank == 0) {
        int stage = 0;
        uint32_t phase = 0, unit = 0, sf_unit = 0;
        const int a_lines = p.a.contract_rows, b_lines = p.b.contract_rows;
        const uint32_t a_step = operand_step(a_lines), b_step = operand_step(b_lines);
        const uint32_t idesc = kFloat ? idesc_f8(kTileM, kTileN) : idesc_mxf8(kTileM, kTileN, a_lines, b_lines);
        bool ok = true;
        for (int item = pair; item < items && ok; item += npairs) {
          const Item it = pair_item(p, item);
          for (int g0 = it.g_begin; g0 < it.g_end && ok; g0 += p.chunk_groups) {
            const int b_begin = 4 * g0, b_end = min(4 * min(it.g_end, g0 + p.chunk_groups), p.a.blocks);
            uint32_t acc = 0;
            if constexpr (!kFloat) {
              const uint32_t buf = unit % S::kBuffers;
              acc = tmem + buf * S::kBufferStep;
              if (!wait_warp(smem_u32(&sh->acc_empty[buf]), ((unit / S::kBuffers) & 1u) ^ 1u, &sh->abort, p.status, 0x810)) { ok = false; break; }
              if (unit && !wait_warp(smem_u32(&sh->overlap), (unit - 1) & 1u, &sh->abort, p.status, 0x811)) { ok = false; break; }
              tc_fence_after();
            }
            for (int b = b_begin; b < b_end; ++b) {
              uint32_t sfa = 0, sfb = 0;
              if constexpr (kFloat) {
                const uint32_t buf = unit % S::kBuffers;
                acc = tmem + buf * S::kBufferStep;
                if (!wait_warp(smem_u32(&sh->acc_empty[buf]), ((unit / S::kBuffers) & 1u) ^ 1u, &sh->abort, p.status, 0x812)) { ok = false; break; }
              } else {
                const uint32_t set = sf_unit & 1u;
                if ((b & 3) == 0 && !wait_warp(smem_u32(&sh->sf_full[set]), (sf_unit >> 1) & 1u, &sh->abort, p.status, 0x813)) { ok = false; break; }
                sfa = tmem + S::kScaleCol + set * 12;
                sfb = sfa + 4;
              }
              if (!wait_warp(smem_u32(&sh->full[stage]), phase, &sh->abort, p.status, 0x820 + stage)) { ok = false; break; }
              tc_fence_after();
              const uint32_t base = smem_u32(tiles + stage * S::kStageBytes);
              const uint64_t da = operand_desc(a_lines, base), db = operand_desc(b_lines, base + S::kABytes);
              const bool last_of_scales = (b & 3) == 3 || b + 1 == b_end;
              if (elect_one()) {
#pragma unroll
                for (uint32_t ks = 0; ks < 4; ++ks) {
                  if constexpr (kFloat)
                    mma_f8_pair(acc, da + ks * a_step, db + ks * b_step, idesc, ks ? 1u : 0u);
                  else
                    mma_mxf8_pair(acc, da + ks * a_step, db + ks * b_step, idesc | idesc_mxf8_block((uint32_t)b & 3u), sfa, sfb, (b > b_begin || ks) ? 1u : 0u);
                }
                mma_commit_pair(smem_u32(&sh->empty[stage]), (uint16_t)3);
                if constexpr (kFloat) {
                  mma_commit_pair(smem_u32(&sh->acc_full[unit % S::kBuffers]), (uint16_t)3);
                } else {
                  if (last_of_scales) mma_commit_pair(smem_u32(&sh->sf_empty[sf_unit & 1u]), (uint16_t)3);
                  if (b + 1 == b_end) mma_commit_pair(smem_u32(&sh->acc_full[unit % S::kBuffers]), (uint16_t)3);
                }
              }
              __syncwarp();
              if (++stage == S::kStages) stage = 0, phase ^= 1u;
              if constexpr (kFloat) ++unit; else sf_unit += last_of_scales;
            }
            if constexpr (!kFloat) ++unit;
          }
        }
        if (sh->abort && elect_one()) {
          mma_commit_pair(smem_u32(&sh->drained), (uint16_t)1);
          const uint64_t t0 = global_timer_ns();
          while (!mbar_try_wait(smem_u32(&sh->drained), 0u) && global_timer_ns() - t0 < kWaitLimitNs) {
          }
        }
      }
    } else if (warp < S::kFirstEpilogue) {
      // ------------------------------ scale words into tensor memory (both CTAs) ------------------------------
      // Row r of an operand's 128 lines is lane r % 32, column r / 32 of its four columns, in every quarter of the lanes:
      // each warp writes the quarter it may touch.  This CTA's 128 lines of A, all 256 of B.
      if constexpr (!kFloat) {
        const uint32_t at = tmem + (((uint32_t)(warp & 3) * 32u) << 16) + S::kScaleCol;
        const uint32_t leader = map_to_cta(smem_u32(&sh->sf_full[0]), 0);
        uint32_t unit = 0;
        bool ok = true;
        for (int item = pair; item < items && ok; item += npairs) {
          const Item it = pair_item(p, item);
          uint32_t wa[4], wb0[4], wb1[4];   // the words of the next group, on their way while this one's are written
          auto fetch = [&](int g) {
            scale_words<4>(p.a, it.m0 + rank * 128, lane, g, wa);
            scale_words<4>(p.b, it.n0, lane, g, wb0);
            scale_words<4>(p.b, it.n0 + 128, lane, g, wb1);
          };
          fetch(it.g_begin);
          for (int g = it.g_begin; g < it.g_end; ++g, ++unit) {
            const uint32_t set = unit & 1u;
            if (!wait_warp(smem_u32(&sh->sf_empty[set]), ((unit >> 1) & 1u) ^ 1u, &sh->abort, p.status, 0x830)) {
              ok = false;
              break;
            }
            tc_fence_after();
            tmem_st_32x4(at + set * 12, wa);
            tmem_st_32x4(at + set * 12 + 4, wb0);
            tmem_st_32x4(at + set * 12 + 8, wb1);
            if (g + 1 < it.g_end) fetch(g + 1);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(leader + set * 8);
          }
        }
      }
    }
  } else {
    if constexpr (kFloat) set_registers_more<S::kEpilogueRegs>();
    // ------------------------------ epilogue (both CTAs) ----------------------------------
    const uint32_t quad = (uint32_t)(warp & 3);
    const int part = (warp - S::kFirstEpilogue) >> 2;   // which 128 of the columns
    uint8_t* box = staging + (warp - S::kFirstEpilogue) * 4096;
    const uint32_t lanes = tmem + ((quad * 32u) << 16);
    const uint32_t empty0 = map_to_cta(smem_u32(&sh->acc_empty[0]), 0), overlap = map_to_cta(smem_u32(&sh->overlap), 0);
    uint32_t unit = 0;
    bool ok = true;
    for (int item = pair; item < items && ok; item += npairs) {
      const Item it = pair_item(p, item);
      const int m = it.m0 + rank * 128 + (int)quad * 32;
      if constexpr (kFloat) {
        const int n = it.n0 + part * 128, row = m + lane;
        const int b_begin = 4 * it.g_begin, b_end = min(4 * it.g_end, p.a.blocks);
        uint64_t acc[64];
#pragma unroll
        for (int e = 0; e < 64; ++e) acc[e] = 0;
        float sa = scale_line_f32(p.a, row, b_begin), sb = scale_tile_f32(p.b, n, b_begin), sa1 = sa, sb1 = sb;
        if (b_begin + 1 < b_end) sa1 = scale_line_f32(p.a, row, b_begin + 1), sb1 = scale_tile_f32(p.b, n, b_begin + 1);
        for (int b = b_begin; b < b_end; ++b, ++unit) {
          const uint32_t buf = unit % S::kBuffers;
          const float s = sa * sb;
          sa = sa1, sb = sb1;
          if (b + 2 < b_end) sa1 = scale_line_f32(p.a, row, b + 2), sb1 = scale_tile_f32(p.b, n, b + 2);
          if (!wait_warp(smem_u32(&sh->acc_full[buf]), (unit / S::kBuffers) & 1u, &sh->abort, p.status, 0x840)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t from = lanes + buf * S::kBufferStep + part * 128;
          const uint64_t s2 = pack_f32x2(s, s);
          uint32_t d[2][32];   // 32 columns are multiplied while the next 32 are read
          tmem_ld_32x32(from, d[0]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tmem_wait_ld();
            if (c < 3) {
              tmem_ld_32x32(from + (c + 1) * 32, d[(c + 1) & 1]);
            } else {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive_cluster(empty0 + buf * 8);
            }
#pragma unroll
            for (int e = 0; e < 32; e += 2) fma_f32x2(acc[c * 16 + e / 2], pack_f32x2(__uint_as_float(d[c & 1][e]), __uint_as_float(d[c & 1][e + 1])), s2);
          }
        }
        if (!ok) break;
        uint32_t w[32];
        constexpr int kPieces = kBf16 ? 2 : 4;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            float lo, hi;
            if constexpr (kBf16) {
              unpack_f32x2(acc[32 * i + e], lo, hi);
              w[e] = pack_bf16(lo, hi);
            } else {
              unpack_f32x2(acc[16 * i + e / 2], lo, hi);
              w[e] = __float_as_uint(e % 2 ? hi : lo);
            }
          }
          store_box<kBf16>(p.out, &map_c, box, lane, w, m, n + i * (128 / kPieces), it.split, p.out.add);
        }
      } else {
        const int n = it.n0 + part * 128;
        for (int g0 = it.g_begin; g0 < it.g_end; g0 += p.chunk_groups, ++unit) {
          const uint32_t buf = unit % S::kBuffers;
          const bool later = g0 > it.g_begin;   // a later range of the same tile is added to the earlier ones
          if (later && p.out.tma && lane == 0) bulk_wait();
          if (!wait_warp(smem_u32(&sh->acc_full[buf]), (unit / S::kBuffers) & 1u, &sh->abort, p.status, 0x841)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t from = lanes + buf * S::kBufferStep + part * 128;
          const bool shared_half = buf == 0 ? part == 1 : part == 0;   // holds the columns that the other accumulator shares
          constexpr int kPieces = kBf16 ? 2 : 4, kWidth = kBf16 ? 64 : 32;
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
            store_box<kBf16>(p.out, &map_c, box, lane, w, m, n + c * kWidth, it.split, p.out.add || later);
          }
        }
      }
    }
    if (lane == 0) bulk_wait();   // the staging memory is read until then
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

// C (+)= the partial sums of the K ranges, added in order.
template <bool kBf16>
__global__ void __launch_bounds__(256) join_kernel(const float* part, int splits, int M, int N, int64_t ld, void* C, int64_t ldc, int add) {
  const int64_t total = (int64_t)M * N, stride = (int64_t)M * ld;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int m = (int)(i / N), n = (int)(i - (int64_t)m * N);
    const float* q = part + (int64_t)m * ld + n;
    float sum = 0.f;
    for (int s = 0; s < splits; ++s) sum += q[s * stride];
    if constexpr (kBf16) {
      static_cast<__nv_bfloat16*>(C)[(int64_t)m * ldc + n] = __float2bfloat16_rn(sum);
    } else {
      float* c = static_cast<float*>(C) + (int64_t)m * ldc + n;
      *c = add ? *c + sum : sum;
    }
  }
}

// ---- few rows of C --------------------------------------------------------------------
constexpr int kMaxCluster = 8;
constexpr int kRowsMost = 128, kRowsMostFloat = 64;   // rows of C in one tile
constexpr int kRowsThreads = 6 * 32;   // producer, issuer, 4 warps for scales and epilogue
template <int NT, bool kFloat>
struct RowsShape {
  static constexpr int kWBytes = 128 * kBlock;
  static constexpr int kStageBytes = kWBytes + NT * kBlock;
  static constexpr int kStages = NT == 128 ? 3 : 4;
  static constexpr int kSets = 4;                                   // scale words of four groups in flight (UE8M0)
  static constexpr int kBuffers = kFloat ? 4 : 1;                   // accumulators, one per block of 128 (FP32 scales)
  static constexpr int kNeeded = kFloat ? kBuffers * NT : NT + kSets * 8;
  static constexpr int kCols = kNeeded <= 64 ? 64 : kNeeded <= 128 ? 128 : 256;
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 512 + 4 * 2 * NT * 4 + 1024;
  static_assert(NT * 128 * 4 <= kStages * kStageBytes, "the partial sums are exchanged in the stages' memory");
};
struct __align__(8) RowsShared {
  uint64_t full[4], empty[4], sf_full[4], sf_empty[4], acc_full[4], acc_empty[4], drained;
  uint32_t tmem_base;
  volatile int abort;
};
static_assert(sizeof(RowsShared) <= 512, "room reserved behind the stages");

__device__ __forceinline__ float4 load_cluster_f32x4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}

// p.a: the rows of C, NT at a time (the instruction's column side), p.b: the lines that become its 128 rows.
template <int NT, bool kFloat, class T>
__global__ void __launch_bounds__(kRowsThreads)
product_rows_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ ProductParams p) {
  using S = RowsShape<NT, kFloat>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  RowsShared* sh = reinterpret_cast<RowsShared*>(tiles + S::kStages * S::kStageBytes);
  float* block_scales = reinterpret_cast<float*>(tiles + S::kStages * S::kStageBytes + 512);   // [warp][2][NT]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank(), size = (int)cluster_size();
  // tiles of rows of C run fastest: the clusters that read the same lines of B do so at about the same time
  const int tile = (int)(blockIdx.x / size), m0 = tile % p.tiles_m * NT, n0 = tile / p.tiles_m * 128;
  const int rows = min(NT, p.out.M - m0);
  const int g_begin = (int)((int64_t)rank * p.groups / size), g_end = (int)((int64_t)(rank + 1) * p.groups / size);
  const int b_begin = 4 * g_begin, b_end = min(4 * g_end, p.a.blocks);

  if (threadIdx.x == 0) {
    prefetch_tensormap(&map_x);
    prefetch_tensormap(&map_w);
    for (int s = 0; s < 4; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1), mbar_init(smem_u32(&sh->empty[s]), 1);
      mbar_init(smem_u32(&sh->sf_full[s]), 4), mbar_init(smem_u32(&sh->sf_empty[s]), 1);
      mbar_init(smem_u32(&sh->acc_full[s]), 1), mbar_init(smem_u32(&sh->acc_empty[s]), 4);
    }
    mbar_init(smem_u32(&sh->drained), 1);
    sh->abort = 0;
    fence_barrier_init();
    fence_proxy_async();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&sh->tmem_base), S::kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh->tmem_base;
  float* sums = reinterpret_cast<float*>(tiles);   // [NT][128] once the operands have been consumed

  if (warp == 0) {
    if (lane == 0) {
      int issued = 0;
      for (int b = b_begin; b < b_end; ++b, ++issued) {
        const int stage = issued % S::kStages;
        if (!wait_bounded(smem_u32(&sh->empty[stage]), ((uint32_t)(issued / S::kStages) & 1u) ^ 1u, &sh->abort, p.status, 0x900 + stage)) break;
        const uint32_t dst = smem_u32(tiles + stage * S::kStageBytes), full = smem_u32(&sh->full[stage]);
        mbar_arrive_expect_tx(full, S::kStageBytes);
        int x, y;
        tile_at(p.b.contract_rows, n0, b, x, y);
        tma_load_2d(dst, &map_w, full, x, y);
        tile_at(p.a.contract_rows, m0, b, x, y);
        tma_load_2d(dst + S::kWBytes, &map_x, full, x, y);
      }
      if (sh->abort) {   // copies in flight land before this CTA leaves
        const uint64_t t0 = global_timer_ns();
        for (int j = max(0, issued - S::kStages); j < issued; ++j)
          while (!mbar_try_wait(smem_u32(&sh->full[j % S::kStages]), (uint32_t)(j / S::kStages) & 1u) && global_timer_ns() - t0 < kWaitLimitNs) {
          }
      }
    }
  } else if (warp == 1) {
    {
      const int w_lines = p.b.contract_rows, x_lines = p.a.contract_rows;
      const uint32_t w_step = operand_step(w_lines), x_step = operand_step(x_lines);
      const uint32_t idesc = kFloat ? idesc_f8(128, NT) : idesc_mxf8(128, NT, w_lines, x_lines);
      for (int b = b_begin; b < b_end; ++b) {
        const int i = b - b_begin, stage = i % S::kStages, buf = i % S::kBuffers, set = (i / 4) % S::kSets;
        if (kFloat && !wait_warp(smem_u32(&sh->acc_empty[buf]), ((uint32_t)(i / S::kBuffers) & 1u) ^ 1u, &sh->abort, p.status, 0x910)) break;
        if (!kFloat && i % 4 == 0 && !wait_warp(smem_u32(&sh->sf_full[set]), (uint32_t)(i / 4 / S::kSets) & 1u, &sh->abort, p.status, 0x911)) break;
        if (!wait_warp(smem_u32(&sh->full[stage]), (uint32_t)(i / S::kStages) & 1u, &sh->abort, p.status, 0x920 + stage)) break;
        tc_fence_after();
        const uint32_t base = smem_u32(tiles + stage * S::kStageBytes);
        const uint64_t dw = operand_desc(w_lines, base), dx = operand_desc(x_lines, base + S::kWBytes);
        if (elect_one()) {
#pragma unroll
          for (uint32_t ks = 0; ks < 4; ++ks) {
            if constexpr (kFloat)
              mma_f8(tmem + buf * NT, dw + ks * w_step, dx + ks * x_step, idesc, ks ? 1u : 0u);
            else
              mma_mxf8(tmem, dw + ks * w_step, dx + ks * x_step, idesc | idesc_mxf8_block((uint32_t)b & 3u), tmem + NT + set * 8, tmem + NT + set * 8 + 4, (i || ks) ? 1u : 0u);
          }
          mma_commit(smem_u32(&sh->empty[stage]));
          if (kFloat || b + 1 == b_end) mma_commit(smem_u32(&sh->acc_full[kFloat ? buf : 0]));
          if (!kFloat && (i % 4 == 3 || b + 1 == b_end)) mma_commit(smem_u32(&sh->sf_empty[set]));
        }
        __syncwarp();
      }
      if (sh->abort && elect_one()) {
        mma_commit(smem_u32(&sh->drained));
        const uint64_t t0 = global_timer_ns();
        while (!mbar_try_wait(smem_u32(&sh->drained), 0u) && global_timer_ns() - t0 < kWaitLimitNs) {
        }
      }
    }
  } else {
    const uint32_t quad = (uint32_t)(warp & 3);
    const uint32_t lanes = tmem + ((quad * 32u) << 16);
    const int line = (int)quad * 32 + lane;   // of the 128
    bool ok = true;
    if constexpr (kFloat) {
      float acc[NT];
#pragma unroll
      for (int e = 0; e < NT; ++e) acc[e] = 0.f;
      float* mine = block_scales + (warp - 2) * 2 * NT;
      constexpr int kPer = (NT + 31) / 32;
      float sx[kPer], sw = scale_tile_f32(p.b, n0, b_begin);
#pragma unroll
      for (int j = 0; j < kPer; ++j) sx[j] = lane + 32 * j < NT ? scale_line_f32(p.a, m0 + lane + 32 * j, b_begin) : 0.f;
      for (int b = b_begin; b < b_end; ++b) {
        const int i = b - b_begin, buf = i % S::kBuffers;
        float* s = mine + (i & 1) * NT;   // two, so that one barrier of the warp is enough
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (lane + 32 * j < NT) s[lane + 32 * j] = sx[j] * sw;
        __syncwarp();
        if (b + 1 < b_end) {
          sw = scale_tile_f32(p.b, n0, b + 1);
#pragma unroll
          for (int j = 0; j < kPer; ++j) sx[j] = lane + 32 * j < NT ? scale_line_f32(p.a, m0 + lane + 32 * j, b + 1) : 0.f;
        }
        if (!wait_warp(smem_u32(&sh->acc_full[buf]), (uint32_t)(i / S::kBuffers) & 1u, &sh->abort, p.status, 0x930)) {
          ok = false;
          break;
        }
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < NT / 16; ++c) {
          uint32_t d[16];
          tmem_ld_32x16(lanes + buf * NT + c * 16, d);
          tmem_wait_ld();
          if (c == NT / 16 - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->acc_empty[buf]));
          }
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 f = *reinterpret_cast<const float4*>(s + c * 16 + e);
            acc[c * 16 + e] = fmaf(__uint_as_float(d[e]), f.x, acc[c * 16 + e]);
            acc[c * 16 + e + 1] = fmaf(__uint_as_float(d[e + 1]), f.y, acc[c * 16 + e + 1]);
            acc[c * 16 + e + 2] = fmaf(__uint_as_float(d[e + 2]), f.z, acc[c * 16 + e + 2]);
            acc[c * 16 + e + 3] = fmaf(__uint_as_float(d[e + 3]), f.w, acc[c * 16 + e + 3]);
          }
        }
      }
      // every warp has seen the last block: all operands have been consumed, their memory takes the sums
      asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
      for (int e = 0; e < NT; ++e) sums[e * 128 + line] = acc[e];
    } else {
      for (int g = g_begin; g < g_end; ++g) {
        const int i = g - g_begin, set = i % S::kSets;
        uint32_t ww[4], wx[4];
        scale_words<4>(p.b, n0, lane, g, ww);
        scale_words<(NT + 31) / 32>(p.a, m0, lane, g, wx);
        if (!wait_warp(smem_u32(&sh->sf_empty[set]), ((uint32_t)(i / S::kSets) & 1u) ^ 1u, &sh->abort, p.status, 0x931)) {
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
      if (ok) ok = wait_warp(smem_u32(&sh->acc_full[0]), 0u, &sh->abort, p.status, 0x932);
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
  for (int e = rank * kRowsThreads + (int)threadIdx.x; e < rows * 32; e += size * kRowsThreads) {
    const int n = n0 + e % 32 * 4, left = p.out.N - n;
    if (left <= 0) continue;
    float4 v[kMaxCluster];
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r)
      if (r < size) v[r] = load_cluster_f32x4(map_to_cta(local + (uint32_t)e * 16u, (uint32_t)r));
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r)
      if (r < size) sum[0] += v[r].x, sum[1] += v[r].y, sum[2] += v[r].z, sum[3] += v[r].w;
    T* c = static_cast<T*>(p.out.ptr) + (int64_t)(m0 + e / 32) * p.out.ld + n;
    if (sizeof(T) == 2 && p.out.tma && left >= 4) {
      *reinterpret_cast<uint2*>(c) = make_uint2(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]));
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < left) store_element(c + k, p.out.add ? load_element(c + k) + sum[k] : sum[k]);
    }
  }
  cluster_arrive_relaxed();   // no CTA leaves while another reads its sums; nothing was written that another waits for
  cluster_wait();
}

// ---- host side ------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static std::atomic<EncodeTiledFn> fn{nullptr};
  EncodeTiledFn f = fn.load(std::memory_order_acquire);
  if (!f) {
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess) return nullptr;
    f = reinterpret_cast<EncodeTiledFn>(sym);
    fn.store(f, std::memory_order_release);
  }
  return f;
}
// cuTensorMapEncodeTiled, which wants a current context: a host thread whose first CUDA call this is has none until the runtime makes the
// device's primary context current.
bool encode(CUtensorMap* map, CUtensorMapDataType type, uint32_t rank, void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
            CUtensorMapL2promotion promotion) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint32_t estr[3] = {1, 1, 1};
  auto call = [&] { return fn(map, type, rank, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE); };
  CUresult r = call();
  if (r == CUDA_ERROR_INVALID_CONTEXT || r == CUDA_ERROR_NOT_INITIALIZED) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(dev) != cudaSuccess) return false;
    r = call();
  }
  return r == CUDA_SUCCESS;
}
// Tiles of an operand: `lines` x 128 values of k, rows of 128 bytes along k (or along the lines).  What lies outside reads as zero.
bool operand_map(CUtensorMap* map, const Operand& o, int64_t K, int lines) {
  const cuuint64_t dims[2] = {(cuuint64_t)(o.contract_rows ? o.lines : K), (cuuint64_t)(o.contract_rows ? K : o.lines)};
  const cuuint64_t strides[1] = {(cuuint64_t)o.ld};
  const cuuint32_t box[2] = {(cuuint32_t)kBlock, (cuuint32_t)(o.contract_rows ? kBlock : lines)};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(o.codes), dims, strides, box, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}
bool output_map(CUtensorMap* map, const Output& o, bool bf16, int splits) {
  const cuuint64_t size = bf16 ? 2 : 4;
  const cuuint64_t dims[3] = {(cuuint64_t)o.N, (cuuint64_t)o.M, (cuuint64_t)splits};
  const cuuint64_t strides[2] = {(cuuint64_t)o.ld * size, (cuuint64_t)o.ld * size * (cuuint64_t)o.M};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / size), 32, 1};
  return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, o.ptr, dims, strides, box, CU_TENSOR_MAP_L2_PROMOTION_NONE);
}

constexpr int kMaxDevices = 64;
// Raises a kernel's dynamic shared memory once per device, and checks its registers.
template <class K>
bool raise_smem(K kernel, size_t bytes, std::atomic<bool> (&done)[kMaxDevices], int registers = 0) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
  if (done[dev].load(std::memory_order_acquire)) return true;
  if (registers) {   // the kernel redistributes this many registers per thread: a build with fewer would wait for them
    cudaFuncAttributes a;
    if (cudaFuncGetAttributes(&a, kernel) != cudaSuccess || a.numRegs < registers) return false;
  }
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return false;
  done[dev].store(true, std::memory_order_release);
  return true;
}

template <bool kFloat, bool kBf16>
bool launch_pair(const CUtensorMap& map_a, const CUtensorMap& map_b, const CUtensorMap& map_c, const ProductParams& p, int pairs, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto kernel = product_pair_kernel<kFloat, kBf16>;
  if (!raise_smem(kernel, PairShape<kFloat>::kSmem, done, kFloat ? PairShape<kFloat>::kLaunchRegs : 0)) return false;
  kernel<<<(unsigned)(2 * pairs), PairShape<kFloat>::kThreads, PairShape<kFloat>::kSmem, st>>>(map_a, map_b, map_c, p);
  return cudaGetLastError() == cudaSuccess;
}

template <int NT, bool kFloat, class T>
bool launch_rows(const CUtensorMap& map_x, const CUtensorMap& map_w, const ProductParams& p, int tiles, int cluster, cudaStream_t st) {
  static std::atomic<bool> done[kMaxDevices];
  auto kernel = product_rows_kernel<NT, kFloat, T>;
  if (!raise_smem(kernel, RowsShape<NT, kFloat>::kSmem, done)) return false;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * cluster), 1, 1);
  cfg.blockDim = dim3(kRowsThreads, 1, 1);
  cfg.dynamicSmemBytes = RowsShape<NT, kFloat>::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, map_x, map_w, p) == cudaSuccess;
}
template <int NT>
bool launch_rows_as(bool floats, bool bf16, const CUtensorMap& map_x, const CUtensorMap& map_w, const ProductParams& p, int tiles, int cluster, cudaStream_t st) {
  if constexpr (NT <= kRowsMostFloat) {   // one accumulator a thread for each of the NT columns
    if (floats)
      return bf16 ? launch_rows<NT, true, __nv_bfloat16>(map_x, map_w, p, tiles, cluster, st) : launch_rows<NT, true, float>(map_x, map_w, p, tiles, cluster, st);
  }
  return bf16 ? launch_rows<NT, false, __nv_bfloat16>(map_x, map_w, p, tiles, cluster, st) : launch_rows<NT, false, float>(map_x, map_w, p, tiles, cluster, st);
}

bool check_operand(const ozk_fp8_operand* o, int64_t lines, int64_t k, Operand* out) {
  const int64_t cols = o->contract_rows ? lines : k;
  if (!o->codes || !o->scales || !aligned16(o->codes) || o->ld % 16 || o->ld < cols) return false;
  if (o->scale_kind < OZK_SCALE_LINES || o->scale_kind > OZK_SCALE_TILES_F32) return false;
  if (o->contract_rows != 0 && o->contract_rows != 1) return false;
  if (o->scale_kind != OZK_SCALE_TILES && (reinterpret_cast<uintptr_t>(o->scales) & 3)) return false;
  *out = Operand{o->codes, o->ld, o->scales, o->scale_kind, o->contract_rows, (int)lines, (int)ceil_div(k, kBlock), ceil_div(cols, kBlock)};
  return true;
}

constexpr size_t kGemmStatusBytes = 1024;
constexpr size_t kGemmWorkspace = 24u << 20;   // status, and the partial sums of at most one tile per CTA pair (74 x 256 KiB)

// How product_rows_kernel would run: NT rows of C a tile, `cluster` CTAs along K.
struct RowsPlan {
  int NT, tiles_m, tiles_n, cluster;
};
RowsPlan rows_plan(const ProductParams& p, bool floats, bool f32_result, int sms) {
  RowsPlan r;
  const int most = floats ? kRowsMostFloat : kRowsMost;
  // an A summed over its rows comes in rows of 128 lines
  r.NT = p.a.contract_rows ? 128 : p.out.M <= 16 ? 16 : p.out.M <= 32 ? 32 : p.out.M <= 64 ? 64 : most;
  r.tiles_m = (int)ceil_div(p.out.M, r.NT);
  r.tiles_n = (int)ceil_div(p.out.N, 128);
  // two CTAs fit a multiprocessor: K is split over a cluster while that fills them
  const int64_t tiles = (int64_t)r.tiles_m * r.tiles_n;
  int c = tiles >= 2 * sms ? 1 : (int)(2 * sms / tiles);
  if (f32_result && c * kRowsRangeGroups < p.groups) c = (int)ceil_div(p.groups, kRowsRangeGroups);   // FP32 results: short ranges
  if (c > p.groups) c = p.groups;
  r.cluster = c > kMaxCluster ? kMaxCluster : c;
  return r;
}
ozk_status run_rows(ProductParams p, const RowsPlan& r, int64_t K, bool floats, bool bf16, cudaStream_t st) {
  CUtensorMap map_x, map_w;
  if (!operand_map(&map_x, p.a, K, r.NT) || !operand_map(&map_w, p.b, K, 128)) return OZK_ERR_CUDA;
  p.tiles_m = r.tiles_m, p.tiles_n = r.tiles_n;
  const int tiles = r.tiles_m * r.tiles_n;
  bool ok;
  switch (r.NT) {
    case 16: ok = launch_rows_as<16>(floats, bf16, map_x, map_w, p, tiles, r.cluster, st); break;
    case 32: ok = launch_rows_as<32>(floats, bf16, map_x, map_w, p, tiles, r.cluster, st); break;
    case 64: ok = launch_rows_as<64>(floats, bf16, map_x, map_w, p, tiles, r.cluster, st); break;
    default: ok = launch_rows_as<128>(floats, bf16, map_x, map_w, p, tiles, r.cluster, st); break;
  }
  return ok ? OZK_OK : OZK_ERR_CUDA;
}

// Which kernel, and how it divides the work.
struct Plan {
  bool rows;
  RowsPlan r;
  int64_t tiles_m, tiles_n;   // of the pairs
  int splits;
  size_t scratch;             // partial sums of the splits in device memory
};
Plan product_plan(const ProductParams& p, bool floats, bool bf16, int sms) {
  Plan q = {};
  q.r = rows_plan(p, floats, !bf16, sms);
  q.tiles_m = ceil_div(p.out.M, kTileM), q.tiles_n = ceil_div(p.out.N, kTileN);
  const int64_t pair_tiles = q.tiles_m * q.tiles_n, row_ctas = (int64_t)q.r.tiles_m * q.r.tiles_n * q.r.cluster;
  // product_rows_kernel where it keeps more of the GPU busy than pairs of CTAs with 256 x 256 tiles would:
  //   UE8M0: up to 128 rows, or while the pairs have tiles for half of them at most (and would split K and join).  Rows against pairs, us:
  //     256 x 4096 x 4096 13.7 : 19.2, 512 x 4096 x 4096 17.9 : 24.9, 1024 x 2048 x 2048 13.7 : 21.4, but 384 x 8192 x 4096 (64 tiles) 26.4 : 18.3.
  //   FP32 scales: one tile of rows, or CTAs that all run at once with at most 8 blocks each, which take longer to scale than to form:
  //     128 x 4096 x 4096 13.6 : 16.9, 512 x 1024 x 4096 12.9 : 15.6, but 512 x 2048 x 8192 (32 blocks) 33 : 23.
  const bool few = floats ? q.r.tiles_m == 1 || (row_ctas <= 2 * sms && 4 * ceil_div(p.groups, q.r.cluster) <= 8)
                          : p.out.M <= kRowsMost || 2 * pair_tiles <= sms / 2;
  const bool ranges_fit = bf16 || (int64_t)q.r.cluster * kRowsRangeGroups >= p.groups;
  q.rows = few && ranges_fit;
  q.splits = 1;
  if (q.rows) return q;
  // fewer tiles than half the pairs: split K so that each pair has one range of at least 1024
  const int pairs = sms / 2;
  if (pair_tiles * 2 <= pairs) {
    q.splits = (int)(pairs / pair_tiles);
    if (q.splits > p.groups / 2) q.splits = p.groups / 2;
    if (q.splits < 1) q.splits = 1;
  }
  if (q.splits > 1) q.scratch = (size_t)q.splits * p.out.M * (size_t)round_up(p.out.N, 4) * 4;
  return q;
}

ozk_status run_pair(ProductParams p, const Plan& plan, int64_t K, bool floats, bool bf16, void* scratch, cudaStream_t st) {
  const int64_t tm = plan.tiles_m, tn = plan.tiles_n;
  if (tm * tn > INT32_MAX) return OZK_ERR_UNSUPPORTED;
  const int pairs = device_sm_count() / 2;
  const int splits = plan.splits;
  p.tiles_m = (int)tm, p.tiles_n = (int)tn;
  const Output c = p.out;
  p.splits = splits;
  const bool out_bf16 = bf16 && splits == 1;
  p.chunk_groups = out_bf16 || floats ? p.groups : kRangeGroups;
  if (splits > 1) {   // rows of whole 16-byte pieces, the last one's zeros included
    const int ld = (int)round_up(c.N, 4);
    p.out = Output{scratch, ld, c.M, ld, 0, 1};
  }
  CUtensorMap map_a, map_b, map_c;
  if (!operand_map(&map_a, p.a, K, 128) || !operand_map(&map_b, p.b, K, kTileN / 2)) return OZK_ERR_CUDA;
  if (p.out.tma) {
    if (!output_map(&map_c, p.out, out_bf16, splits)) return OZK_ERR_CUDA;
  } else {
    map_c = map_a;   // not used
  }
  const int64_t items = tm * tn * splits;
  if (items > INT32_MAX) return OZK_ERR_UNSUPPORTED;
  const int grid = (int)(items < pairs ? items : pairs);
  const bool ok = floats ? (out_bf16 ? launch_pair<true, true>(map_a, map_b, map_c, p, grid, st) : launch_pair<true, false>(map_a, map_b, map_c, p, grid, st))
                         : (out_bf16 ? launch_pair<false, true>(map_a, map_b, map_c, p, grid, st) : launch_pair<false, false>(map_a, map_b, map_c, p, grid, st));
  if (!ok) return OZK_ERR_CUDA;
  if (splits > 1) {
    const int64_t blocks = ceil_div((int64_t)c.M * c.N, 256);
    const int64_t most = (int64_t)device_sm_count() * 16;
    const unsigned g = (unsigned)(blocks < most ? blocks : most);
    const float* part = static_cast<const float*>(p.out.ptr);
    if (bf16)
      join_kernel<true><<<g, 256, 0, st>>>(part, splits, c.M, c.N, p.out.ld, c.ptr, c.ld, 0);
    else
      join_kernel<false><<<g, 256, 0, st>>>(part, splits, c.M, c.N, p.out.ld, c.ptr, c.ld, c.add);
    if (cudaGetLastError() != cudaSuccess) return OZK_ERR_CUDA;
  }
  return OZK_OK;
}

}  // namespace
}  // namespace ozk

using namespace ozk;

namespace {

// Arguments that do not depend on where the results go.
ozk_status check_product(int64_t M, int64_t N, int64_t K, const ozk_fp8_operand* A, const ozk_fp8_operand* B, int c_type, ProductParams* p, bool* floats) {
  if (M < 0 || N < 0 || K < 0 || !A || !B || (c_type != OZK_F32 && c_type != OZK_BF16)) return OZK_ERR_INVALID_ARG;
  if (M > INT32_MAX || N > INT32_MAX || K > INT32_MAX) return OZK_ERR_UNSUPPORTED;
  Operand a = {}, b = {};
  if (K > 0 && M > 0 && N > 0 && (!check_operand(A, M, K, &a) || !check_operand(B, N, K, &b))) return OZK_ERR_INVALID_ARG;
  *floats = a.kind >= OZK_SCALE_LINES_F32 || b.kind >= OZK_SCALE_LINES_F32;
  if (*floats && (a.kind != OZK_SCALE_LINES_F32 || b.kind != OZK_SCALE_TILES_F32 || a.contract_rows || b.contract_rows))
    return OZK_ERR_UNSUPPORTED;
  *p = ProductParams{};
  p->a = a, p->b = b;
  p->out.M = (int)M, p->out.N = (int)N;
  p->splits = 1;
  p->groups = (int)ceil_div(K, kGroupK);
  return OZK_OK;
}

}  // namespace

extern "C" {

size_t ozk_fp8_gemm_workspace_bytes(void) { return kGemmWorkspace; }

ozk_status ozk_fp8_gemm_plan(int64_t M, int64_t N, int64_t K, const ozk_fp8_operand* A, const ozk_fp8_operand* B, int c_type, int sms, ozk_fp8_plan* plan) {
  ProductParams p;
  bool floats;
  const ozk_status rc = check_product(M, N, K, A, B, c_type, &p, &floats);
  if (rc != OZK_OK) return rc;
  if (!plan || sms < 0) return OZK_ERR_INVALID_ARG;
  *plan = ozk_fp8_plan{};
  if (M == 0 || N == 0 || K == 0) return OZK_OK;
  if (sms == 0) sms = device_sm_count();
  if (sms < 2) return OZK_ERR_CUDA;
  const Plan q = product_plan(p, floats, c_type == OZK_BF16, sms);
  plan->pairs = q.rows ? 0 : 1;
  plan->tile_rows = q.rows ? q.r.NT : kTileM;
  plan->tile_cols = q.rows ? 128 : kTileN;
  plan->tiles = q.rows ? (int64_t)q.r.tiles_m * q.r.tiles_n : q.tiles_m * q.tiles_n;
  plan->splits = q.rows ? q.r.cluster : q.splits;
  plan->scratch_bytes = q.scratch;
  return OZK_OK;
}

ozk_status ozk_fp8_gemm_scratch(int64_t M, int64_t N, int64_t K, const ozk_fp8_operand* A, const ozk_fp8_operand* B, void* C, int c_type,
                                int64_t ldc, int accumulate, void* status, void* scratch, size_t scratch_bytes, void* stream) {
  ProductParams p;
  bool floats;
  const ozk_status rc = check_product(M, N, K, A, B, c_type, &p, &floats);
  if (rc != OZK_OK) return rc;
  if (ldc < N || (accumulate != 0 && accumulate != 1)) return OZK_ERR_INVALID_ARG;
  if (accumulate && c_type != OZK_F32) return OZK_ERR_UNSUPPORTED;
  if (M == 0 || N == 0) return OZK_OK;
  if (!C || (reinterpret_cast<uintptr_t>(C) & (c_type == OZK_F32 ? 3 : 1))) return OZK_ERR_INVALID_ARG;
  if (!status) return OZK_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(status) & 255) || (reinterpret_cast<uintptr_t>(scratch) & 255)) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool bf16 = c_type == OZK_BF16;
  const size_t size = bf16 ? 2 : 4;
  if (K == 0) {   // an empty sum
    if (!accumulate && cudaMemset2DAsync(C, (size_t)ldc * size, 0, (size_t)N * size, (size_t)M, st) != cudaSuccess) return OZK_ERR_CUDA;
    return OZK_OK;
  }
  p.out = Output{C, ldc, (int)M, (int)N, accumulate, aligned16(C) && ((size_t)ldc * size) % 16 == 0 ? 1 : 0};
  p.status = static_cast<StatusBlock*>(status);
  const int sms = device_sm_count();
  if (sms < 2) return OZK_ERR_CUDA;
  const Plan plan = product_plan(p, floats, bf16, sms);
  if (plan.rows) return run_rows(p, plan.r, K, floats, bf16, st);
  if (plan.scratch > 0 && (!scratch || scratch_bytes < plan.scratch)) return OZK_ERR_WORKSPACE;   // before anything is enqueued
  return run_pair(p, plan, K, floats, bf16, scratch, st);
}

ozk_status ozk_fp8_gemm(int64_t M, int64_t N, int64_t K, const ozk_fp8_operand* A, const ozk_fp8_operand* B, void* C, int c_type,
                        int64_t ldc, int accumulate, void* workspace, size_t workspace_size, void* stream) {
  if (!workspace) workspace = workspace_ptr(), workspace_size = workspace_bytes();
  uint8_t* ws = workspace_size < kGemmWorkspace ? nullptr : static_cast<uint8_t*>(workspace);
  return ozk_fp8_gemm_scratch(M, N, K, A, B, C, c_type, ldc, accumulate, ws, ws ? ws + kGemmStatusBytes : nullptr, ws ? kGemmWorkspace - kGemmStatusBytes : 0, stream);
}

}  // extern "C"
