// Quantisation to E4M3 with one power-of-two scale per block of 128 elements.
//
//   scale = 2^ceil(log2(amax / 448)), code = E4M3(x / scale): the division is exact, so both the scale and the code are
//   determined bit for bit, whatever the order of the maximum.
//
// One pass over X for both orientations.  16384 x 8192 BF16 on one B200: by rows 73 us (5.5 TB/s), by columns 69 us (5.9), both 100 us
// (5.4), by tiles 61 us (6.6); 8190 x 4100 FP32 by tiles 31 us (5.4).  Bound by memory, and with both orientations by instructions too.
#include "ozk_fp8.cuh"

namespace ozk {
namespace {

using namespace fp8;

// ---- 128 x 128 tiles ------------------------------------------------------------------
// A tile per thread block, held in registers as it lies in memory: it is read once for both orientations.  Thread t has, of
// rows t / 8 + 32 i, the 16 bytes from byte (t % 8) * 16 of every 128: eight lanes read whole 128-byte lines.
// Magnitudes are compared as integers, two BF16 at a time; what is not finite shows as the largest of them, and then the
// block looks again without it.
template <class T>
struct Words;
template <>
struct Words<__nv_bfloat16> {
  static constexpr int kPiece = 8, kPieces = 2, kWords = 4;   // elements and words per 16 bytes, pieces per row of the tile
  __device__ static __forceinline__ uint32_t magnitude(uint32_t w) { return w & 0x7FFF7FFFu; }
  __device__ static __forceinline__ uint32_t finite_magnitude(uint32_t w) {
    const uint32_t a = w & 0x7FFF7FFFu;
    return ((a & 0xFFFFu) < 0x7F80u ? a & 0xFFFFu : 0u) | (a < 0x7F800000u ? a & 0xFFFF0000u : 0u);
  }
  __device__ static __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ static __forceinline__ uint32_t float_bits(uint32_t m, int i) { return i ? m & 0xFFFF0000u : m << 16; }   // element i of a word
  __device__ static __forceinline__ uint32_t largest(uint32_t m) { return max(m << 16, m & 0xFFFF0000u); }
  __device__ static __forceinline__ float value(const uint32_t* w, int e) { return e % 2 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]); }
};
template <>
struct Words<float> {
  static constexpr int kPiece = 4, kPieces = 4, kWords = 4;
  __device__ static __forceinline__ uint32_t magnitude(uint32_t w) { return w & 0x7FFFFFFFu; }
  __device__ static __forceinline__ uint32_t finite_magnitude(uint32_t w) { return finite_bits(__uint_as_float(w)); }
  __device__ static __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
  __device__ static __forceinline__ uint32_t float_bits(uint32_t m, int) { return m; }
  __device__ static __forceinline__ uint32_t largest(uint32_t m) { return m; }
  __device__ static __forceinline__ float value(const uint32_t* w, int e) { return __uint_as_float(w[e]); }
};

// 16 bytes of a row, zeros beyond `left` elements.  kVec: what the row's place and stride allow (kSingle, kWhole: 16 bytes at once, kWordly: 4 bytes).
enum { kSingle = 0, kWhole = 1, kWordly = 2 };
template <class T, int kVec>
__device__ __forceinline__ void load_piece(const T* p, int left, uint32_t* w) {
  constexpr int kPiece = Words<T>::kPiece;
  if (kVec == kWhole && left >= kPiece) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else if (kVec == kWordly && left >= kPiece) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __ldg(reinterpret_cast<const uint32_t*>(p) + i);
  } else {
    w[0] = w[1] = w[2] = w[3] = 0;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
      if (i >= left) continue;
      if constexpr (sizeof(T) == 2) w[i / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i % 2));
      else w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    }
  }
}
// Its codes: x times reciprocals of scales, which may differ from column to column; `bad`: NaN for what is not finite.
template <class T>
__device__ __forceinline__ void store_piece(uint8_t* q, int left, const uint32_t* w, const Pair* recip, int step, bool bad) {
  constexpr int kPiece = Words<T>::kPiece;
  uint32_t out[kPiece / 4];
#pragma unroll
  for (int k = 0; k < kPiece / 4; ++k) {
    float2 y[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float a = Words<T>::value(w, 4 * k + 2 * h), b = Words<T>::value(w, 4 * k + 2 * h + 1);
      const Pair r = recip[(2 * k + h) * step];
      y[h] = both(pair(a, b) * r);
      if (bad) y[h] = make_float2(scaled(a, both(r).x), scaled(b, both(r).y));
    }
    out[k] = pack4(y[0].x, y[0].y, y[1].x, y[1].y);
  }
  if (left >= kPiece) {
    if constexpr (kPiece == 8) *reinterpret_cast<uint2*>(q) = make_uint2(out[0], out[1]); else *reinterpret_cast<uint32_t*>(q) = out[0];
  } else {
#pragma unroll
    for (int i = 0; i < kPiece; ++i)
      if (i < left) q[i] = (uint8_t)(out[i / 4] >> (8 * (i % 4)));
  }
}

// By rows: a warp takes 512 columns (one word of scales) of kR rows, all loaded before the first is reduced.  Each 16-byte
// piece of a lane lies beside its neighbours'; 16 lanes (BF16) or all 32 (FP32) hold a block.  The warps of a thread block take
// consecutive rows, whose words of scales are neighbours: single words far apart cost more than the codes.
template <class T, bool kVec, int kR>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* X, int64_t ldx, int rows, int cols, uint8_t* Q, int64_t ldq, uint32_t* S) {
  using W = Words<T>;
  constexpr int kPiece = W::kPiece, kPieces = 512 / (32 * kPiece), kLanes = kBlock / kPiece;
  const int64_t strips = (rows + kR - 1) / kR, item = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const int g = (int)(item / strips), r0 = (int)(item % strips) * kR, lane = threadIdx.x % 32;
  if ((int64_t)g * 512 >= cols) return;
  const int c0 = g * 512 + lane * kPiece;
  uint32_t x[kR][kPieces][4];
#pragma unroll
  for (int i = 0; i < kR; ++i)
#pragma unroll
    for (int q = 0; q < kPieces; ++q)
      load_piece<T, kVec>(X + (int64_t)(r0 + i) * ldx + c0 + q * 32 * kPiece, r0 + i < rows ? cols - c0 - q * 32 * kPiece : 0, x[i][q]);
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    uint32_t word = 0;
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      const uint32_t* w = x[i][q];
      uint32_t top = W::largest(W::larger(W::larger(W::magnitude(w[0]), W::magnitude(w[1])), W::larger(W::magnitude(w[2]), W::magnitude(w[3]))));
      const bool bad = __any_sync(0xFFFFFFFFu, top >= 0x7F800000u);
      if (bad)
        top = W::largest(W::larger(W::larger(W::finite_magnitude(w[0]), W::finite_magnitude(w[1])), W::larger(W::finite_magnitude(w[2]), W::finite_magnitude(w[3]))));
#pragma unroll
      for (int d = 1; d < kLanes; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
      const uint32_t c = scale_code(top);
      const Pair recip = pair(scale_recip(c), scale_recip(c));
      const int left = cols - c0 - q * 32 * kPiece;
      if (left > 0 && r0 + i < rows) store_piece<T>(Q + (int64_t)(r0 + i) * ldq + c0 + q * 32 * kPiece, left, w, &recip, 0, bad);
      if constexpr (kLanes == 16) word |= (c | __shfl_down_sync(0xFFFFFFFFu, c, 16) << 8) << (16 * q); else word |= c << (8 * q);
    }
    if (lane == 0 && r0 + i < rows) S[(int64_t)g * rows + r0 + i] = word;
  }
}

// Ranges of rows whose blocks of 128 begin with each of them: tile row tr is a block of the segments, and the codes by columns lie
// block after block, with zeros behind the rows of a segment's last one.  A product that sums over the rows of one segment then needs no masks, and
// starts where a box of it may start.  16384 x 4096 BF16 in 16 segments, both ways: 57 us (4.6 TB/s), bound by memory and, at the start of each
// thread block, by the search for its segment.
struct Segments {
  const int* offsets;
  int count;
};
// First row of block `index`, and how many rows of its segment are left from there (0: there is no such block).  Offsets are held within the rows and
// never fall.  By one warp.
__device__ __forceinline__ int2 segment_block(const Segments& s, int rows, int index, int lane) {
  int carry = 0, top = min(max(__ldg(s.offsets), 0), rows);
  for (int e0 = 0; e0 < s.count; e0 += 32) {
    int f = e0 + lane < s.count ? min(max(__ldg(s.offsets + e0 + lane + 1), top), rows) : top;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, f, d);
      if (lane >= d) f = max(f, v);
    }
    int b = __shfl_up_sync(0xFFFFFFFFu, f, 1);
    if (lane == 0) b = top;
    const int blocks = (f - b + kBlock - 1) / kBlock;
    int sum = blocks;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, sum, d);
      if (lane >= d) sum += v;
    }
    const uint32_t beyond = __ballot_sync(0xFFFFFFFFu, index < carry + sum);
    if (beyond) {
      const int first = b + (index - carry - sum + blocks) * kBlock, l = __ffs(beyond) - 1;
      return make_int2(__shfl_sync(0xFFFFFFFFu, first, l), __shfl_sync(0xFFFFFFFFu, f - first, l));
    }
    carry += __shfl_sync(0xFFFFFFFFu, sum, 31);
    top = __shfl_sync(0xFFFFFFFFu, f, 31);
  }
  return make_int2(0, 0);
}

// kTiles: blockIdx.y is one of several matrices, x_step and q_step apart.
template <class T, int kVec, bool kRows, bool kCols, bool kTiles, bool kSegments = false>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) quantize_tile_kernel(const T* X, int64_t ldx, int rows, int cols, uint8_t* Qr, int64_t ldr, uint8_t* Sr,
                                                            uint8_t* Qc, int64_t ldc, uint8_t* Sc, Segments segments = {}, int64_t x_step = 0, int64_t q_step = 0) {
  using W = Words<T>;
  constexpr int kPiece = W::kPiece, kPieces = W::kPieces, kWords = W::kWords, kRowWords = kPieces * kWords;   // words per thread and row
  constexpr int kTileWords = kRowWords * 8;
  __shared__ __align__(16) uint32_t part[8][kCols ? kTileWords : 1];
  __shared__ __align__(16) float column_recip[kCols ? kBlock : 1];
  __shared__ uint32_t tile_top[8], row_code[kRows ? kBlock : 1];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, c = lane % 8;
  const int tiles_c = (cols + kBlock - 1) / kBlock, tiles_r = (rows + kBlock - 1) / kBlock;
  const int tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  int first = tr * kBlock, live = rows - first;   // the tile's first row of X, and the rows from there on
  if constexpr (kSegments) {
    __shared__ int2 block;
    if (warp == 0) {
      const int2 found = segment_block(segments, rows, tr, lane);
      if (lane == 0) block = found;
    }
    __syncthreads();
    first = block.x, live = block.y;
    if (live == 0) return;
  }
  if constexpr (kTiles) X += blockIdx.y * x_step, Qc += blockIdx.y * q_step, Sc += blockIdx.y * (int64_t)tiles_r * tiles_c;
  const int r_in = threadIdx.x / 8, r0 = first + r_in, c0 = tc * kBlock + c * kPiece;
  uint32_t x[4][kRowWords];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      const int col = c0 + q * 8 * kPiece;
      load_piece<T, kVec>(X + (int64_t)(r0 + 32 * i) * ldx + col, r_in + 32 * i < live ? cols - col : 0, &x[i][q * kWords]);
    }
  // largest magnitudes of this thread's rows and columns
  uint32_t row_top[4], col_top[kRowWords];
  auto look = [&](auto magnitude) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t a[kRowWords];
#pragma unroll
      for (int k = 0; k < kRowWords; ++k) {
        a[k] = magnitude(x[i][k]);
        col_top[k] = i ? W::larger(col_top[k], a[k]) : a[k];
      }
      uint32_t top = a[0];
#pragma unroll
      for (int k = 1; k < kRowWords; ++k) top = W::larger(top, a[k]);
      row_top[i] = W::largest(top);
    }
  };
  look([](uint32_t w) { return W::magnitude(w); });
  const bool bad = __syncthreads_or(max(max(row_top[0], row_top[1]), max(row_top[2], row_top[3])) >= 0x7F800000u);
  if (bad) look([](uint32_t w) { return W::finite_magnitude(w); });

  if constexpr (kCols) {
#pragma unroll
    for (int k = 0; k < kRowWords; ++k) {
      col_top[k] = W::larger(col_top[k], __shfl_xor_sync(0xFFFFFFFFu, col_top[k], 8));
      col_top[k] = W::larger(col_top[k], __shfl_xor_sync(0xFFFFFFFFu, col_top[k], 16));
    }
    if (lane < 8) {
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
        *reinterpret_cast<uint4*>(&part[warp][(q * 8 + c) * kWords]) = make_uint4(col_top[q * 4], col_top[q * 4 + 1], col_top[q * 4 + 2], col_top[q * 4 + 3]);
    }
  }
  if constexpr (kTiles) {
    const uint32_t t = __reduce_max_sync(0xFFFFFFFFu, max(max(row_top[0], row_top[1]), max(row_top[2], row_top[3])));
    if (lane == 0) tile_top[warp] = t;
  }
  // the four rows' pieces, by reciprocals that belong to the row or to the columns
  auto store = [&](uint8_t* Q, int64_t ld, int row, int most, auto recip_of, int step) {   // the first `most` rows of the tile from `row` on
    uint8_t* at = Q + (int64_t)(row + r_in) * ld + c0;
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      const int col = q * 8 * kPiece;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Pair* recip = recip_of(q, i);
        if (r_in + 32 * i < most && c0 + col < cols)
          store_piece<T>(at + (int64_t)(32 * i) * ld + col, cols - c0 - col, &x[i][q * kWords], recip, step, bad);
      }
    }
  };
  if constexpr (kRows) {
    Pair recip[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t top = row_top[i];
#pragma unroll
      for (int d = 1; d < 8; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
      const uint32_t code = scale_code(top);
      recip[i] = pair(scale_recip(code), scale_recip(code));
      if (c == 0) row_code[threadIdx.x / 8 + 32 * i] = code;
    }
    store(Qr, ldr, first, live, [&](int, int i) { return &recip[i]; }, 0);
  }
  __syncthreads();
  if constexpr (kRows) {   // a warp's 32 scale bytes in one request
    const int i = (int)threadIdx.x - kBlock, r = first + i;
    if (i >= 0 && i < live) {
      uint8_t* s = Sr + ((int64_t)(tc / 4) * rows + r) * 4;
      s[tc % 4] = (uint8_t)row_code[i];
      if (tc + 1 == tiles_c)
        for (int b = tc % 4 + 1; b < 4; ++b) s[b] = 127;
    }
  }
  if constexpr (kCols || kTiles) {
    float tile_recip = 0.f;
    if constexpr (kTiles) {
      uint32_t t = tile_top[0];
#pragma unroll
      for (int w = 1; w < 8; ++w) t = max(t, tile_top[w]);
      const uint32_t code = scale_code(t);
      tile_recip = scale_recip(code);
      if (threadIdx.x == 0) Sc[(int64_t)tr * tiles_c + tc] = (uint8_t)code;
    } else {
      if (threadIdx.x < kTileWords) {
        constexpr int kPerWord = kPiece / kWords;
        uint32_t t = part[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < 8; ++w) t = W::larger(t, part[w][threadIdx.x]);
#pragma unroll
        for (int k = 0; k < kPerWord; ++k) {
          const int col = (int)threadIdx.x * kPerWord + k;
          const uint32_t code = scale_code(W::float_bits(t, k));
          column_recip[col] = scale_recip(code);
          if (tc * kBlock + col < cols) {
            uint8_t* s = Sc + ((int64_t)(tr / 4) * cols + tc * kBlock + col) * 4;
            s[tr % 4] = (uint8_t)code;
            if (!kSegments && tr + 1 == tiles_r)
              for (int b = tr % 4 + 1; b < 4; ++b) s[b] = 127;
          }
        }
      }
      __syncthreads();
    }
    Pair recip[kTiles ? 1 : kPieces * kPiece / 2];
    if constexpr (kTiles) {
      recip[0] = pair(tile_recip, tile_recip);
    } else {
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
#pragma unroll
        for (int k = 0; k < kPiece / 2; ++k) {
          const float2 f = *reinterpret_cast<const float2*>(&column_recip[(q * 8 + c) * kPiece + 2 * k]);
          recip[q * kPiece / 2 + k] = pair(f.x, f.y);
        }
    }
    store(Qc, ldc, kSegments ? tr * kBlock : first, kSegments ? kBlock : live, [&](int q, int) { return &recip[kTiles ? 0 : q * kPiece / 2]; }, kTiles ? 0 : 1);
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

// Four rows a warp once that still leaves every multiprocessor 16 warps; one row a warp where there are few, for the latency.
template <class T, bool kVec>
cudaError_t launch_rows(int rows, int cols, const T* X, int64_t ldx, uint8_t* Q, int64_t ld, uint32_t* S, cudaStream_t st) {
  const int64_t groups = ceil_div(cols, 512);
  if (groups * ceil_div(rows, 4) >= (int64_t)device_sm_count() * 16)
    quantize_rows_kernel<T, kVec, 4><<<(unsigned)ceil_div(groups * ceil_div(rows, 4), 8), 256, 0, st>>>(X, ldx, rows, cols, Q, ld, S);
  else
    quantize_rows_kernel<T, kVec, 1><<<(unsigned)ceil_div(groups * rows, 8), 256, 0, st>>>(X, ldx, rows, cols, Q, ld, S);
  return cudaGetLastError();
}

template <class T, bool kVec>
cudaError_t launch_lines(int rows, int cols, const T* X, int64_t ldx, uint8_t* Qr, int64_t ldr, uint8_t* Sr, uint8_t* Qc, int64_t ldc, uint8_t* Sc,
                         cudaStream_t st) {
  const int64_t tiles = ceil_div(rows, kBlock) * ceil_div(cols, kBlock);
  if (!Qc) return launch_rows<T, kVec>(rows, cols, X, ldx, Qr, ldr, reinterpret_cast<uint32_t*>(Sr), st);
  if (Qr)
    quantize_tile_kernel<T, kVec, true, true, false><<<(unsigned)tiles, 256, 0, st>>>(X, ldx, rows, cols, Qr, ldr, Sr, Qc, ldc, Sc);
  else
    quantize_tile_kernel<T, kVec, false, true, false><<<(unsigned)tiles, 256, 0, st>>>(X, ldx, rows, cols, nullptr, 0, nullptr, Qc, ldc, Sc);
  return cudaGetLastError();
}
template <class T, bool kVec>
cudaError_t launch_tiles(int count, int rows, int cols, const T* X, int64_t ldx, int64_t x_step, uint8_t* Q, int64_t ld, int64_t q_step, uint8_t* S, cudaStream_t st) {
  const dim3 grid((unsigned)(ceil_div(rows, kBlock) * ceil_div(cols, kBlock)), (unsigned)count);
  quantize_tile_kernel<T, kVec, false, false, true><<<grid, 256, 0, st>>>(X, ldx, rows, cols, nullptr, 0, nullptr, Q, ld, S, Segments{}, x_step, q_step);
  return cudaGetLastError();
}
template <class T, int kVec>
cudaError_t launch_segments(int64_t blocks, const Segments& s, int rows, int cols, const T* X, int64_t ldx, uint8_t* Qr, int64_t ldr, uint8_t* Sr, uint8_t* Qc, int64_t ldc,
                            uint8_t* Sc, cudaStream_t st) {
  const unsigned tiles = (unsigned)(blocks * ceil_div(cols, kBlock));
  if (Qr) quantize_tile_kernel<T, kVec, true, true, false, true><<<tiles, 256, 0, st>>>(X, ldx, rows, cols, Qr, ldr, Sr, Qc, ldc, Sc, s);
  else quantize_tile_kernel<T, kVec, false, true, false, true><<<tiles, 256, 0, st>>>(X, ldx, rows, cols, nullptr, 0, nullptr, Qc, ldc, Sc, s);
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

ozk_status ozk_fp8_quantize_segments(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, const int32_t* offsets, int64_t segments,
                                     uint8_t* row_codes, int64_t row_ld, uint8_t* row_scales, uint8_t* col_codes, int64_t col_ld, uint8_t* col_scales, void* stream) {
  bool vec;
  const ozk_status rc = check_input(rows, cols, X, x_type, ldx, &vec);
  if (rc != OZK_OK) return rc;
  if (segments < 0) return OZK_ERR_INVALID_ARG;
  if (segments > INT32_MAX - 1024) return OZK_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0 || segments == 0) return OZK_OK;
  const int64_t blocks = ozk_fp8_segment_blocks(rows, segments);
  if (blocks * kBlock > INT32_MAX || blocks * ceil_div(cols, kBlock) > INT32_MAX) return OZK_ERR_UNSUPPORTED;   // rows of the blocks are ints too, up to 127 a segment more
  if (!offsets || (reinterpret_cast<uintptr_t>(offsets) & 3)) return OZK_ERR_INVALID_ARG;
  if ((row_codes || row_scales) && !good_codes(row_codes, row_ld, cols, row_scales, 4)) return OZK_ERR_INVALID_ARG;
  if (!good_codes(col_codes, col_ld, cols, col_scales, 4)) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const Segments s{offsets, (int)segments};
  const int r = (int)rows, c = (int)cols;
  cudaError_t e;
  if (x_type == OZK_F32) {
    const float* x = static_cast<const float*>(X);
    e = vec ? launch_segments<float, kWhole>(blocks, s, r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st)
            : launch_segments<float, kSingle>(blocks, s, r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st);
  } else {
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(X);
    // rows of an odd multiple of two elements, 9001 x 4100: 4 bytes at once 41 us, single elements 76
    const bool wordly = (reinterpret_cast<uintptr_t>(X) & 3) == 0 && ldx % 2 == 0;
    e = vec ? launch_segments<__nv_bfloat16, kWhole>(blocks, s, r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st)
        : wordly ? launch_segments<__nv_bfloat16, kWordly>(blocks, s, r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st)
                 : launch_segments<__nv_bfloat16, kSingle>(blocks, s, r, c, x, ldx, row_codes, row_ld, row_scales, col_codes, col_ld, col_scales, st);
  }
  return e == cudaSuccess ? OZK_OK : OZK_ERR_CUDA;
}

ozk_status ozk_fp8_quantize_tiles(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, uint8_t* codes, int64_t ld, uint8_t* scales,
                                  void* stream) {
  return ozk_fp8_quantize_experts(1, rows, cols, X, x_type, ldx, 0, codes, ld, 0, scales, stream);
}

ozk_status ozk_fp8_quantize_experts(int64_t experts, int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, int64_t x_step, uint8_t* codes, int64_t ld,
                                    int64_t step, uint8_t* scales, void* stream) {
  bool vec;
  const ozk_status rc = check_input(rows, cols, X, x_type, ldx, &vec);
  if (rc != OZK_OK) return rc;
  if (experts < 0 || step % 16 || (experts > 1 && (x_step < 0 || step < (rows - 1) * ld + cols))) return OZK_ERR_INVALID_ARG;
  if (experts > 65535) return OZK_ERR_UNSUPPORTED;
  if (experts == 0 || rows == 0 || cols == 0) return OZK_OK;
  if (!good_codes(codes, ld, cols, scales, 1)) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  vec = vec && (x_step * (x_type == OZK_F32 ? 4 : 2)) % 16 == 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int n = (int)experts, r = (int)rows, c = (int)cols;
  cudaError_t e;
  if (x_type == OZK_F32) {
    const float* x = static_cast<const float*>(X);
    e = vec ? launch_tiles<float, true>(n, r, c, x, ldx, x_step, codes, ld, step, scales, st) : launch_tiles<float, false>(n, r, c, x, ldx, x_step, codes, ld, step, scales, st);
  } else {
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(X);
    e = vec ? launch_tiles<__nv_bfloat16, true>(n, r, c, x, ldx, x_step, codes, ld, step, scales, st)
            : launch_tiles<__nv_bfloat16, false>(n, r, c, x, ldx, x_step, codes, ld, step, scales, st);
  }
  return e == cudaSuccess ? OZK_OK : OZK_ERR_CUDA;
}

}  // extern "C"
