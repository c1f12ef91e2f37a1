// Quantisation to E4M3 with one power-of-two scale per block of 128 elements.
//
//   scale = 2^ceil(log2(amax / 448)), code = E4M3(x / scale): the division is exact, so both the scale and the code are
//   determined bit for bit, whatever the order of the maximum.
#include "ozk_fp8.cuh"

namespace ozk {
namespace {

using namespace fp8;

// 16 consecutive elements of a row from column c on; zeros beyond `left` elements.
template <class T, bool kVec>
__device__ __forceinline__ void load16(const T* p, int left, float (&x)[16]) {
  if (left <= 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
  } else if (kVec && left >= 16) {
    if constexpr (sizeof(T) == 2) {
      const uint4* q = reinterpret_cast<const uint4*>(p);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 w = __ldg(q + h);
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[8 * h + 2 * i] = bf16_lo(v[i]), x[8 * h + 2 * i + 1] = bf16_hi(v[i]);
      }
    } else {
      const float4* q = reinterpret_cast<const float4*>(p);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const float4 w = __ldg(q + h);
        x[4 * h] = w.x, x[4 * h + 1] = w.y, x[4 * h + 2] = w.z, x[4 * h + 3] = w.w;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i < left ? load_element(p + i) : 0.f;
  }
}
// 16 codes at a 16-byte aligned address; only the first `left` of them inside the matrix.
__device__ __forceinline__ void store16(uint8_t* p, int left, const uint32_t (&w)[4]) {
  if (left >= 16) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < left) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// By rows: one warp per 512 columns of a row (one word of scales).  Eight lanes of 16 elements hold a block.
template <class T, bool kVec>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* X, int64_t ldx, int rows, int cols, uint8_t* Q, int64_t ldq, uint32_t* S) {
  const int64_t groups = (cols + 511) / 512;
  const int64_t item = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (item >= groups * rows) return;
  const int g = (int)(item / rows), r = (int)(item % rows), lane = threadIdx.x % 32;
  const int c0 = g * 512 + lane * 16;
  float x[16];
  load16<T, kVec>(X + (int64_t)r * ldx + c0, cols - c0, x);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, finite_bits(x[i]));
#pragma unroll
  for (int d = 1; d < 8; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
  const uint32_t c = scale_code(top);
  const float recip = scale_recip(c);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack4(scaled(x[4 * i], recip), scaled(x[4 * i + 1], recip), scaled(x[4 * i + 2], recip), scaled(x[4 * i + 3], recip));
  if (cols - c0 > 0) store16(Q + (int64_t)r * ldq + c0, cols - c0, w);
  uint32_t word = c;
  word |= __shfl_sync(0xFFFFFFFFu, c, 8) << 8;
  word |= __shfl_sync(0xFFFFFFFFu, c, 16) << 16;
  word |= __shfl_sync(0xFFFFFFFFu, c, 24) << 24;
  if (lane == 0) S[(int64_t)g * rows + r] = word;
}

// A 128 x 128 tile per block: thread (t / 8, t % 8) holds 16 columns of rows t / 8 + 32 i.
template <class T, bool kVec, bool kRows, bool kCols, bool kTiles>
__global__ void __launch_bounds__(256) quantize_tile_kernel(const T* X, int64_t ldx, int rows, int cols, uint8_t* Qr, int64_t ldr, uint8_t* Sr,
                                                            uint8_t* Qc, int64_t ldc, uint8_t* Sc) {
  __shared__ uint32_t part[8][kBlock], tile_top[4];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int tiles_c = (cols + kBlock - 1) / kBlock, tiles_r = (rows + kBlock - 1) / kBlock;
  const int tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  const int r0 = tr * kBlock + threadIdx.x / 8, c0 = tc * kBlock + (threadIdx.x % 8) * 16;
  float x[4][16];
#pragma unroll
  for (int i = 0; i < 4; ++i) load16<T, kVec>(X + (int64_t)(r0 + 32 * i) * ldx + c0, r0 + 32 * i < rows ? cols - c0 : 0, x[i]);
  if constexpr (kRows) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) top = max(top, finite_bits(x[i][j]));
#pragma unroll
      for (int d = 1; d < 8; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
      const int r = r0 + 32 * i;
      if (r >= rows) continue;
      const uint32_t c = scale_code(top);
      const float recip = scale_recip(c);
      if (cols > c0) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = pack4(scaled(x[i][4 * j], recip), scaled(x[i][4 * j + 1], recip), scaled(x[i][4 * j + 2], recip), scaled(x[i][4 * j + 3], recip));
        store16(Qr + (int64_t)r * ldr + c0, cols - c0, w);
      }
      if (lane % 8 == 0) {
        uint8_t* s = Sr + ((int64_t)(tc / 4) * rows + r) * 4;
        s[tc % 4] = (uint8_t)c;
        if (tc + 1 == tiles_c)
          for (int b = tc % 4 + 1; b < 4; ++b) s[b] = 127;
      }
    }
  }
  if constexpr (kCols || kTiles) {
    uint32_t top[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      top[j] = max(max(finite_bits(x[0][j]), finite_bits(x[1][j])), max(finite_bits(x[2][j]), finite_bits(x[3][j])));
      top[j] = max(top[j], __shfl_xor_sync(0xFFFFFFFFu, top[j], 8));
      top[j] = max(top[j], __shfl_xor_sync(0xFFFFFFFFu, top[j], 16));
    }
    if (lane < 8) {
#pragma unroll
      for (int j = 0; j < 16; ++j) part[warp][lane * 16 + j] = top[j];
    }
    __syncthreads();
    if (threadIdx.x < kBlock) {
      uint32_t t = part[0][threadIdx.x];
#pragma unroll
      for (int w = 1; w < 8; ++w) t = max(t, part[w][threadIdx.x]);
      if constexpr (kTiles) {
        t = __reduce_max_sync(0xFFFFFFFFu, t);
        if (lane == 0) tile_top[warp] = t;
      } else {
        part[0][threadIdx.x] = scale_code(t);
      }
    }
    __syncthreads();
    uint32_t tile_code = 0;
    if constexpr (kTiles) {
      tile_code = scale_code(max(max(tile_top[0], tile_top[1]), max(tile_top[2], tile_top[3])));
      if (threadIdx.x == 0) Sc[(int64_t)tr * tiles_c + tc] = (uint8_t)tile_code;
    } else if (threadIdx.x < kBlock && tc * kBlock + threadIdx.x < cols) {
      uint8_t* s = Sc + ((int64_t)(tr / 4) * cols + tc * kBlock + threadIdx.x) * 4;
      s[tr % 4] = (uint8_t)part[0][threadIdx.x];
      if (tr + 1 == tiles_r)
        for (int b = tr % 4 + 1; b < 4; ++b) s[b] = 127;
    }
    if (cols > c0) {
      float recip[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) recip[j] = scale_recip(kTiles ? tile_code : part[0][c0 - tc * kBlock + j]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = r0 + 32 * i;
        if (r >= rows) break;
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = pack4(scaled(x[i][4 * j], recip[4 * j]), scaled(x[i][4 * j + 1], recip[4 * j + 1]), scaled(x[i][4 * j + 2], recip[4 * j + 2]),
                       scaled(x[i][4 * j + 3], recip[4 * j + 3]));
        store16(Qc + (int64_t)r * ldc + c0, cols - c0, w);
      }
    }
  }
}

constexpr int64_t kMaxExtent = INT32_MAX - 1024;   // column and row indexes are ints, with room for the last tile

ozk_status check_input(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, bool* vec) {
  if (rows < 0 || cols < 0 || (x_type != OZK_F32 && x_type != OZK_BF16) || ldx < cols) return OZK_ERR_INVALID_ARG;
  if (rows > kMaxExtent || cols > kMaxExtent) return OZK_ERR_UNSUPPORTED;
  if (ceil_div(rows, kBlock) * ceil_div(cols, kBlock) > INT32_MAX) return OZK_ERR_UNSUPPORTED;
  const int size = x_type == OZK_F32 ? 4 : 2;
  if (rows > 0 && cols > 0 && (!X || (reinterpret_cast<uintptr_t>(X) & (size - 1)))) return OZK_ERR_INVALID_ARG;
  *vec = aligned16(X) && (ldx * size) % 16 == 0;   // 16-byte loads; single elements otherwise
  return OZK_OK;
}
bool good_codes(const uint8_t* q, int64_t ld, int64_t cols, const void* scales, int scale_align) {
  return q && scales && aligned16(q) && ld % 16 == 0 && ld >= cols && (reinterpret_cast<uintptr_t>(scales) & (scale_align - 1)) == 0;
}

template <class T, bool kVec>
cudaError_t launch_lines(int rows, int cols, const T* X, int64_t ldx, uint8_t* Qr, int64_t ldr, uint8_t* Sr, uint8_t* Qc, int64_t ldc, uint8_t* Sc,
                         cudaStream_t st) {
  const int64_t tiles = ceil_div(rows, kBlock) * ceil_div(cols, kBlock);
  if (!Qc)
    quantize_rows_kernel<T, kVec><<<(unsigned)ceil_div((int64_t)rows * ceil_div(cols, 512), 8), 256, 0, st>>>(X, ldx, rows, cols, Qr, ldr,
                                                                                                        reinterpret_cast<uint32_t*>(Sr));
  else if (Qr)
    quantize_tile_kernel<T, kVec, true, true, false><<<(unsigned)tiles, 256, 0, st>>>(X, ldx, rows, cols, Qr, ldr, Sr, Qc, ldc, Sc);
  else
    quantize_tile_kernel<T, kVec, false, true, false><<<(unsigned)tiles, 256, 0, st>>>(X, ldx, rows, cols, nullptr, 0, nullptr, Qc, ldc, Sc);
  return cudaGetLastError();
}
template <class T, bool kVec>
cudaError_t launch_tiles(int rows, int cols, const T* X, int64_t ldx, uint8_t* Q, int64_t ld, uint8_t* S, cudaStream_t st) {
  const int64_t tiles = ceil_div(rows, kBlock) * ceil_div(cols, kBlock);
  quantize_tile_kernel<T, kVec, false, false, true><<<(unsigned)tiles, 256, 0, st>>>(X, ldx, rows, cols, nullptr, 0, nullptr, Q, ld, S);
  return cudaGetLastError();
}

}  // namespace
}  // namespace ozk

using namespace ozk;

extern "C" {

size_t ozk_fp8_line_scale_bytes(int64_t lines, int64_t k) {
  if (lines < 0 || k < 0) return 0;
  return (size_t)fp8::ceil_div(k, 4 * fp8::kBlock) * (size_t)lines * 4;
}

ozk_status ozk_fp8_quantize_lines(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, uint8_t* row_codes, int64_t row_ld,
                                  uint8_t* row_scales, uint8_t* col_codes, int64_t col_ld, uint8_t* col_scales, void* stream) {
  bool vec;
  const ozk_status rc = check_input(rows, cols, X, x_type, ldx, &vec);
  if (rc != OZK_OK) return rc;
  if (rows == 0 || cols == 0) return OZK_OK;
  const bool by_rows = row_codes || row_scales, by_cols = col_codes || col_scales;
  if (!by_rows && !by_cols) return OZK_ERR_INVALID_ARG;
  if (by_rows && !good_codes(row_codes, row_ld, cols, row_scales, 4)) return OZK_ERR_INVALID_ARG;
  if (by_cols && !good_codes(col_codes, col_ld, cols, col_scales, 4)) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int r = (int)rows, c = (int)cols;
  cudaError_t e;
  if (x_type == OZK_F32) {
    const float* x = static_cast<const float*>(X);
    e = vec ? launch_lines<float, true>(r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st)
            : launch_lines<float, false>(r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st);
  } else {
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(X);
    e = vec ? launch_lines<__nv_bfloat16, true>(r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st)
            : launch_lines<__nv_bfloat16, false>(r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st);
  }
  return e == cudaSuccess ? OZK_OK : OZK_ERR_CUDA;
}

ozk_status ozk_fp8_quantize_tiles(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, uint8_t* codes, int64_t ld, uint8_t* scales,
                                  void* stream) {
  bool vec;
  const ozk_status rc = check_input(rows, cols, X, x_type, ldx, &vec);
  if (rc != OZK_OK) return rc;
  if (rows == 0 || cols == 0) return OZK_OK;
  if (!good_codes(codes, ld, cols, scales, 1)) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int r = (int)rows, c = (int)cols;
  cudaError_t e;
  if (x_type == OZK_F32) {
    const float* x = static_cast<const float*>(X);
    e = vec ? launch_tiles<float, true>(r, c, x, ldx, codes, ld, scales, st) : launch_tiles<float, false>(r, c, x, ldx, codes, ld, scales, st);
  } else {
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(X);
    e = vec ? launch_tiles<__nv_bfloat16, true>(r, c, x, ldx, codes, ld, scales, st)
            : launch_tiles<__nv_bfloat16, false>(r, c, x, ldx, codes, ld, scales, st);
  }
  return e == cudaSuccess ? OZK_OK : OZK_ERR_CUDA;
}

}  // extern "C"
