// What the block-scaled products share: operands and their scale words, results that leave by boxes, tensor maps.
#pragma once

#include <cuda.h>

#include <atomic>

#include "ozk_fp8.cuh"
#include "ozk_ptx.cuh"

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

constexpr int kGroupK = 4 * kBlock;            // elements of K that a word of scales serves
constexpr int kRangeGroups = 8192 / kGroupK;   // FP32 results: longest range summed by the tensor cores alone

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
  // a row at a time, consecutive lanes, consecutive elements; eight rows' sums are read before the first is written (133 rows of 29 experts, 5029 x 670 added in
  // FP32: 167 us, one by one 274)
  const int rows = min(32, o.M - m);
  for (int r0 = 0; r0 < rows; r0 += 8) {
    uint32_t v[8];
    float sum[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int r = r0 + k;   // up to 31: the staging has them all
      v[k] = *reinterpret_cast<const uint32_t*>(staging + r * 128 + (((lane / 4) ^ (r & 7)) * 16) + (lane % 4) * 4);
      if constexpr (!kBf16) sum[k] = add && r < rows && n + lane < o.N ? static_cast<const float*>(o.ptr)[(int64_t)(m + r) * o.ld + n + lane] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (r0 + k >= rows) break;
      const int64_t at = (int64_t)(m + r0 + k) * o.ld;
      if constexpr (kBf16) {
        uint16_t* c = static_cast<uint16_t*>(o.ptr) + at;
        if (n + 2 * lane < o.N) c[n + 2 * lane] = (uint16_t)v[k];
        if (n + 2 * lane + 1 < o.N) c[n + 2 * lane + 1] = (uint16_t)(v[k] >> 16);
      } else if (n + lane < o.N) {
        static_cast<float*>(o.ptr)[at + n + lane] = add ? sum[k] + __uint_as_float(v[k]) : __uint_as_float(v[k]);
      }
    }
  }
  __syncwarp();
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
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

}  // namespace
}  // namespace ozk
