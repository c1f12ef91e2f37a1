// RMS norm with the residual's addition, its answer in E4M3 by blocks of 128, and its gradients.
//
//   h = round(x + r) in the type of r;  s = 1 / sqrt(mean(h^2) + eps);  y = h s w;  codes and scales of y as the quantiser's.
//   g = dy w;  dx = dh + s (g - h s mean(g h s));  dw = sum over the rows of dy h s.
// The norm is of h as it is stored, so that the backward pass, which reads h and s, differentiates what was computed.  Sums and all
// arithmetic in FP32, in an order that depends on the sizes alone; y is rounded once, to its codes.
//
// Rows: a row lies in the registers of 1 to 16 warps, 512 columns a warp and step; in each step lane l holds columns 128 b + 4 l .. + 3 (or, where
// the rows do not allow 4 elements at a time, 128 b + 32 i + l) of four blocks b, so that a block's maximum is one warp-wide integer maximum
// and the four scales of a word are known to the whole warp.
// Columns: blocks run along the rows, so a second kernel reads h again, tile by tile, with s known.
#include <type_traits>

#include "ozk_fp8.cuh"

namespace ozk {
namespace {

using namespace fp8;

// ---- four elements of a lane ------------------------------------------------------------
template <class T>
struct Quad {
  uint32_t w[sizeof(T)];   // BF16: two words, FP32: four
};
__device__ __forceinline__ float quad_value(const Quad<__nv_bfloat16>& q, int i) { return i % 2 ? bf16_hi(q.w[i / 2]) : bf16_lo(q.w[i / 2]); }
__device__ __forceinline__ float quad_value(const Quad<float>& q, int i) { return __uint_as_float(q.w[i]); }
// Column of element i of a lane in the block that starts at `c0`, and how far those of a lane are apart.
template <bool kVec>
__device__ __forceinline__ int quad_col(int c0, int lane, int i) { return kVec ? c0 + 4 * lane + i : c0 + 32 * i + lane; }

// Read once, so it need not stay in L1; not through the read-only path, because h may be written over x or r.
__device__ __forceinline__ void load_stream(const __nv_bfloat16* p, Quad<__nv_bfloat16>& q) {
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(q.w[0]), "=r"(q.w[1]) : "l"(p) : "memory");
}
__device__ __forceinline__ void load_stream(const float* p, Quad<float>& q) {
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.w[0]), "=r"(q.w[1]), "=r"(q.w[2]), "=r"(q.w[3]) : "l"(p) : "memory");
}
// The lane's elements of the block at column c0 of a row; zeros beyond `cols`.
template <bool kVec, class T>
__device__ __forceinline__ void load_quad(const T* row, int c0, int lane, int cols, Quad<T>& q) {
  if (kVec && c0 + 4 * lane + 4 <= cols) {
    load_stream(row + c0 + 4 * lane, q);
    return;
  }
#pragma unroll
  for (int k = 0; k < (int)sizeof(T); ++k) q.w[k] = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = quad_col<kVec>(c0, lane, i);
    if (c >= cols) continue;
    if constexpr (sizeof(T) == 2) q.w[i / 2] |= (uint32_t) * reinterpret_cast<const volatile uint16_t*>(row + c) << (16 * (i % 2));
    else q.w[i] = *reinterpret_cast<const volatile uint32_t*>(row + c);
  }
}
template <bool kVec, class T>
__device__ __forceinline__ void store_quad(T* row, int c0, int lane, int cols, const float (&v)[4]) {
  if (kVec && c0 + 4 * lane + 4 <= cols) {
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
      *reinterpret_cast<uint2*>(row + c0 + 4 * lane) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    } else {
      *reinterpret_cast<float4*>(row + c0 + 4 * lane) = make_float4(v[0], v[1], v[2], v[3]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = quad_col<kVec>(c0, lane, i);
    if (c < cols) store_element(row + c, v[i]);
  }
}
// E4M3 codes, which lie at multiples of 16 bytes: four at a time in either layout of x where the lane's columns are neighbours.
template <bool kVec>
__device__ __forceinline__ void store_codes(uint8_t* row, int c0, int lane, int cols, uint32_t codes) {
  if (kVec && c0 + 4 * lane + 4 <= cols) {
    *reinterpret_cast<uint32_t*>(row + c0 + 4 * lane) = codes;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = quad_col<kVec>(c0, lane, i);
    if (c < cols) row[c] = (uint8_t)(codes >> (8 * i));
  }
}
// Weights are read again for every row: they stay in L1, and the registers they would take hold the rows in flight.
template <bool kVec>
__device__ __forceinline__ void load_weight(const void* w, int bf16, int c0, int lane, int cols, float (&v)[4]) {
  if (kVec && c0 + 4 * lane + 4 <= cols) {
    if (bf16) {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(w) + c0 + 4 * lane));
      v[0] = bf16_lo(u.x), v[1] = bf16_hi(u.x), v[2] = bf16_lo(u.y), v[3] = bf16_hi(u.y);
    } else {
      const float4 f = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + c0 + 4 * lane));
      v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = quad_col<kVec>(c0, lane, i);
    v[i] = c >= cols ? 0.f : bf16 ? __bfloat162float(__ldg(static_cast<const __nv_bfloat16*>(w) + c)) : __ldg(static_cast<const float*>(w) + c);
  }
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

constexpr int kGroup = 512;       // columns a warp holds at a time
constexpr int kMostWarps = 16;
constexpr int kMostCols = kGroup * kMostWarps * 4;

// How a row is laid over a thread block: `warps` a row, `rows` of them side by side, V groups of 512 columns a warp.
struct Layout {
  int warps, rows, v;
};
Layout row_layout(int64_t cols, int most_of_one) {
  const int groups = (int)ceil_div(cols, kGroup);
  int v = groups <= most_of_one ? 1 : groups <= 32 ? 2 : 4, warps = 1;
  while (warps * v < groups) warps *= 2;
  return {warps, warps < 8 ? 8 / warps : 1, v};
}
constexpr int kNormOne = 16, kGradOne = 8;   // groups up to which a warp takes one
// Sum over the warps of this thread's row, the same in all of them.  `side` alternates, so that one barrier is enough.
__device__ __forceinline__ float row_sum(float v, float (*part)[kMostWarps], int side, int warps, int warp) {
  v = warp_sum(v);
  if (warps == 1) return v;
  if (threadIdx.x % 32 == 0) part[side][warp] = v;
  __syncthreads();
  const int first = warp & ~(warps - 1);
  v = 0.f;
  for (int i = 0; i < warps; ++i) v += part[side][first + i];
  return v;
}

struct NormParams {
  const void *x, *r, *w;
  void *h, *y;
  int64_t ldx, ldr, ldh, ldy, ldq;
  int rows, cols, w_bf16, warps, side_rows;
  float eps;
  float* root;
  uint8_t* codes;
  uint32_t* scales;
};

struct None {};   // no residual: h is x and is not written
template <class TX, class TR>
struct Stored { using type = TR; };
template <class TX>
struct Stored<TX, None> { using type = TX; };

template <class TX, class TR, bool kVec, int V>
__global__ void __launch_bounds__(512, V == 4 ? 1 : 2) norm_rows_kernel(const __grid_constant__ NormParams p) {
  constexpr bool kAdd = !std::is_same<TR, None>::value;
  using TH = typename Stored<TX, TR>::type;
  __shared__ float part[2][kMostWarps];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, in_row = warp % p.warps, step = p.warps * kGroup;
  const int c_first = in_row * kGroup;
  const int64_t row = (int64_t)blockIdx.x * p.side_rows + warp / p.warps;
  const bool live = row < p.rows;
  float h[V][4][4], sum = 0.f;
  if (live) {
    const TX* px = static_cast<const TX*>(p.x) + row * p.ldx;
    const TH* pr = static_cast<const TH*>(p.r) + row * p.ldr;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c0 = c_first + v * step;
      Quad<TX> x[4];
      Quad<TH> r[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        load_quad<kVec>(px, c0 + q * kBlock, lane, p.cols, x[q]);
        if constexpr (kAdd) load_quad<kVec>(pr, c0 + q * kBlock, lane, p.cols, r[q]);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f = quad_value(x[q], i);
          if constexpr (kAdd) {
            f += quad_value(r[q], i);
            if constexpr (sizeof(TH) == 2) f = __bfloat162float(__float2bfloat16_rn(f));
          }
          h[v][q][i] = f;
          sum = fmaf(f, f, sum);
        }
        if constexpr (kAdd) store_quad<kVec>(static_cast<TH*>(p.h) + row * p.ldh, c0 + q * kBlock, lane, p.cols, h[v][q]);
      }
    }
  }
  sum = row_sum(sum, part, 0, p.warps, warp);
  if (!live) return;
  const float s = __frsqrt_rn(__fdiv_rn(sum, (float)p.cols) + p.eps);
  if (in_row == 0 && lane == 0 && p.root) p.root[row] = s;
  if (!p.codes && !p.y) return;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c0 = c_first + v * step;
    if (c0 >= p.cols) break;
    uint32_t word = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float w[4], (&y)[4] = h[v][q];
      load_weight<kVec>(p.w, p.w_bf16, c0 + q * kBlock, lane, p.cols, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = y[i] * s * w[i];
      if (p.y) store_quad<kVec>(static_cast<TX*>(p.y) + row * p.ldy, c0 + q * kBlock, lane, p.cols, y);
      if (!p.codes) continue;
      const uint32_t top = max(max(finite_bits(y[0]), finite_bits(y[1])), max(finite_bits(y[2]), finite_bits(y[3])));
      const uint32_t c = scale_code(__reduce_max_sync(0xFFFFFFFFu, top));
      const float recip = scale_recip(c);
      store_codes<kVec>(p.codes + row * p.ldq, c0 + q * kBlock, lane, p.cols, pack4(scaled(y[0], recip), scaled(y[1], recip), scaled(y[2], recip), scaled(y[3], recip)));
      word |= c << (8 * q);
    }
    if (p.codes && lane == 0) p.scales[(int64_t)(c0 / kGroup) * p.rows + row] = word;
  }
}

// Codes by columns: a 128 x 128 tile of h a thread block, warp w with rows w + 8 i.
template <class TH, bool kVec>
__global__ void __launch_bounds__(256, sizeof(TH) == 2 ? 4 : 2) norm_cols_kernel(const TH* H, int64_t ldh, const float* root, const void* W, int w_bf16, int rows, int cols,
                                                                               uint8_t* Q, int64_t ldq, uint8_t* S) {
  __shared__ uint32_t part[8][kBlock];
  __shared__ float recips[kBlock], roots[kBlock];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int tiles_c = (cols + kBlock - 1) / kBlock, tiles_r = (rows + kBlock - 1) / kBlock;
  const int tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c, r0 = tr * kBlock, c0 = tc * kBlock;
  Quad<TH> h[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) load_quad<kVec>(H + (int64_t)(r0 + warp + 8 * i) * ldh, c0, lane, r0 + warp + 8 * i < rows ? cols : 0, h[i]);
  if (threadIdx.x < kBlock) roots[threadIdx.x] = r0 + (int)threadIdx.x < rows ? root[r0 + threadIdx.x] : 0.f;
  float w[4];
  load_weight<kVec>(W, w_bf16, c0, lane, cols, w);
  __syncthreads();
  uint32_t top[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float s = roots[warp + 8 * i];
#pragma unroll
    for (int k = 0; k < 4; ++k) top[k] = max(top[k], finite_bits(quad_value(h[i], k) * s * w[k]));
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[warp][quad_col<kVec>(0, lane, k)] = top[k];
  __syncthreads();
  if (threadIdx.x < kBlock) {
    uint32_t t = part[0][threadIdx.x];
#pragma unroll
    for (int i = 1; i < 8; ++i) t = max(t, part[i][threadIdx.x]);
    const uint32_t c = scale_code(t);
    recips[threadIdx.x] = scale_recip(c);
    const int col = c0 + (int)threadIdx.x;
    if (col < cols) {
      uint8_t* s = S + ((int64_t)(tr / 4) * cols + col) * 4;
      s[tr % 4] = (uint8_t)c;
      if (tr + 1 == tiles_r)
        for (int b = tr % 4 + 1; b < 4; ++b) s[b] = 127;
    }
  }
  __syncthreads();
  float recip[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) recip[k] = recips[quad_col<kVec>(0, lane, k)];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = r0 + warp + 8 * i;
    if (r >= rows) break;
    const float s = roots[warp + 8 * i];
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = scaled(quad_value(h[i], k) * s * w[k], recip[k]);
    store_codes<kVec>(Q + (int64_t)r * ldq, c0, lane, cols, pack4(y[0], y[1], y[2], y[3]));
  }
}

// ---- gradients --------------------------------------------------------------------------
struct GradParams {
  const void *dy, *h, *dh, *w;
  void* dx;
  const float* root;
  int64_t lddy, ldh, lddh, lddx;
  int rows, cols, w_bf16, warps, side_rows;
  float* parts;   // [grid x side_rows][cols], or NULL
};

// Rows as in the forward pass.  Each thread adds up its columns' share of dw over the rows it sees; dw_kernel adds the thread blocks' sums.
template <class TD, class TH, bool kVec, int V>
__global__ void __launch_bounds__(V == 1 ? 256 : 512, V == 1 ? 3 : 1) norm_backward_kernel(const __grid_constant__ GradParams p) {
  __shared__ float part[2][kMostWarps];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, in_row = warp % p.warps, step = p.warps * kGroup;
  const int c_first = in_row * kGroup;
  const int64_t stride = (int64_t)gridDim.x * p.side_rows, first = (int64_t)blockIdx.x * p.side_rows + warp / p.warps;
  Quad<TD> d[V][4];
  Quad<TH> h[V][4], e[4];   // e: what is added, fetched early where it has room
  float dw[V][4][4];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) dw[v][q][i] = 0.f;
  const int64_t rounds = (p.rows - (int64_t)blockIdx.x * p.side_rows + stride - 1) / stride;
  int64_t row = first;
  for (int64_t n = 0; n < rounds; ++n, row += stride) {
    const bool live = row < p.rows;
    const float s = live ? p.root[row] : 0.f;
    float sum = 0.f;
    if (live) {
      const TD* pd = static_cast<const TD*>(p.dy) + row * p.lddy;
      const TH* ph = static_cast<const TH*>(p.h) + row * p.ldh;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          load_quad<kVec>(pd, c_first + v * step + q * kBlock, lane, p.cols, d[v][q]);
          load_quad<kVec>(ph, c_first + v * step + q * kBlock, lane, p.cols, h[v][q]);
        }
      if constexpr (V == 1) {
        if (p.dh) {
#pragma unroll
          for (int q = 0; q < 4; ++q) load_quad<kVec>(static_cast<const TH*>(p.dh) + row * p.lddh, c_first + q * kBlock, lane, p.cols, e[q]);
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float w[4];
          load_weight<kVec>(p.w, p.w_bf16, c_first + v * step + q * kBlock, lane, p.cols, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float dy = quad_value(d[v][q], i), hn = quad_value(h[v][q], i) * s;
            dw[v][q][i] = fmaf(dy, hn, dw[v][q][i]);
            sum = fmaf(dy * w[i], hn, sum);
          }
        }
    }
    sum = row_sum(sum, part, (int)(n & 1), p.warps, warp);
    if (!live) continue;
    const float mean = __fdiv_rn(sum, (float)p.cols);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c0 = c_first + v * step + q * kBlock;
        if (c0 >= p.cols) continue;
        float out[4], w[4];
        load_weight<kVec>(p.w, p.w_bf16, c0, lane, p.cols, w);
        if constexpr (V > 1) {
          if (p.dh) load_quad<kVec>(static_cast<const TH*>(p.dh) + row * p.lddh, c0, lane, p.cols, e[q]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float g = quad_value(d[v][q], i) * w[i], hn = quad_value(h[v][q], i) * s;
          out[i] = s * fmaf(-hn, mean, g);
          if (p.dh) out[i] += quad_value(e[q], i);
        }
        store_quad<kVec>(static_cast<TH*>(p.dx) + row * p.lddx, c0, lane, p.cols, out);
      }
  }
  if (!p.parts) return;
  float* mine = p.parts + first * p.cols;   // the first row that this warp saw names its sums
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = quad_col<kVec>(c_first + v * step + q * kBlock, lane, i);
        if (c < p.cols) mine[c] = dw[v][q][i];
      }
}

// dw = the thread blocks' sums, added in a fixed order: 32 columns and 32 strands of rows a thread block.
__global__ void __launch_bounds__(1024) norm_dw_kernel(const float* parts, int count, int cols, float* dw) {
  __shared__ float strand[32][33];
  const int lane = threadIdx.x % 32, s = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int i = s; i < count; i += 32) sum += parts[(int64_t)i * cols + c];
  }
  strand[s][lane] = sum;
  __syncthreads();
  const float v = warp_sum(strand[lane][s]);   // warp s joins the strands of column s
  if (lane == 0 && blockIdx.x * 32 + s < cols) dw[blockIdx.x * 32 + s] = v;
}

// ---- host side ----------------------------------------------------------------------------
bool type_ok(int t) { return t == OZK_F32 || t == OZK_BF16; }
int type_size(int t) { return t == OZK_F32 ? 4 : 2; }
bool on(const void* p, int size) { return p && (reinterpret_cast<uintptr_t>(p) & (size - 1)) == 0; }
// Four elements at a time.
bool quads(const void* p, int64_t ld, int size) { return (reinterpret_cast<uintptr_t>(p) & (4 * size - 1)) == 0 && ld % 4 == 0; }

// Thread blocks of the backward pass: what runs at once, so that there are few partial sums of dw.
int grad_grid(int64_t rows, const Layout& l) {
  const int64_t need = ceil_div(rows, l.rows), room = (int64_t)device_sm_count() * (l.v == 1 ? 3 : l.warps <= 8 ? 2 : 1);
  return (int)(need < room ? need : room);
}

template <class TX, class TR, bool kVec>
void launch_norm_rows(const NormParams& p, const Layout& l, cudaStream_t st) {
  const unsigned grid = (unsigned)ceil_div(p.rows, l.rows), threads = (unsigned)(32 * l.warps * l.rows);
  switch (l.v) {
    case 1: norm_rows_kernel<TX, TR, kVec, 1><<<grid, threads, 0, st>>>(p); break;
    case 2: norm_rows_kernel<TX, TR, kVec, 2><<<grid, threads, 0, st>>>(p); break;
    default: norm_rows_kernel<TX, TR, kVec, 4><<<grid, threads, 0, st>>>(p); break;
  }
}
template <class TX, class TR>
void launch_norm_rows(bool vec, const NormParams& p, const Layout& l, cudaStream_t st) {
  if (vec) launch_norm_rows<TX, TR, true>(p, l, st); else launch_norm_rows<TX, TR, false>(p, l, st);
}
template <class TH>
void launch_norm_cols(bool vec, const void* h, int64_t ldh, const NormParams& p, uint8_t* q, int64_t ldq, uint8_t* s, cudaStream_t st) {
  const unsigned tiles = (unsigned)(ceil_div(p.rows, kBlock) * ceil_div(p.cols, kBlock));
  if (vec)
    norm_cols_kernel<TH, true><<<tiles, 256, 0, st>>>(static_cast<const TH*>(h), ldh, p.root, p.w, p.w_bf16, p.rows, p.cols, q, ldq, s);
  else
    norm_cols_kernel<TH, false><<<tiles, 256, 0, st>>>(static_cast<const TH*>(h), ldh, p.root, p.w, p.w_bf16, p.rows, p.cols, q, ldq, s);
}
template <class TD, class TH, bool kVec>
void launch_backward(const GradParams& p, const Layout& l, int grid, cudaStream_t st) {
  const unsigned threads = (unsigned)(32 * l.warps * l.rows);
  switch (l.v) {
    case 1: norm_backward_kernel<TD, TH, kVec, 1><<<(unsigned)grid, threads, 0, st>>>(p); break;
    case 2: norm_backward_kernel<TD, TH, kVec, 2><<<(unsigned)grid, threads, 0, st>>>(p); break;
    default: norm_backward_kernel<TD, TH, kVec, 4><<<(unsigned)grid, threads, 0, st>>>(p); break;
  }
}
template <class TD, class TH>
void launch_backward(bool vec, const GradParams& p, const Layout& l, int grid, cudaStream_t st) {
  if (vec) launch_backward<TD, TH, true>(p, l, grid, st); else launch_backward<TD, TH, false>(p, l, grid, st);
}

}  // namespace
}  // namespace ozk

using namespace ozk;

extern "C" {

ozk_status ozk_rms_norm(int64_t rows, int64_t cols, const void* X, int x_type, int64_t ldx, const void* R, int r_type, int64_t ldr, void* H, int64_t ldh,
                        const void* weight, int w_type, double eps, float* root, void* Y, int64_t ldy, uint8_t* row_codes, int64_t row_ld,
                        uint8_t* row_scales, uint8_t* col_codes, int64_t col_ld, uint8_t* col_scales, void* stream) {
  if (rows < 0 || cols < 0 || !type_ok(x_type) || !type_ok(w_type) || ldx < cols || !(eps >= 0.0)) return OZK_ERR_INVALID_ARG;
  if (R && (!type_ok(r_type) || ldr < cols || ldh < cols)) return OZK_ERR_INVALID_ARG;
  if (rows > INT32_MAX - 1024 || cols > kMostCols || (R && r_type != x_type && r_type != OZK_F32)) return OZK_ERR_UNSUPPORTED;
  const bool by_rows = row_codes || row_scales, by_cols = col_codes || col_scales;
  if (rows == 0 || cols == 0) return OZK_OK;
  const int h_type = R ? r_type : x_type;
  if (!on(X, type_size(x_type)) || !on(weight, type_size(w_type)) || (R && (!on(R, type_size(r_type)) || !on(H, type_size(r_type))))) return OZK_ERR_INVALID_ARG;
  if (Y && (!on(Y, type_size(x_type)) || ldy < cols)) return OZK_ERR_INVALID_ARG;
  if ((root && !on(root, 4)) || (by_cols && !root)) return OZK_ERR_INVALID_ARG;
  if (by_rows && (!row_codes || !row_scales || !aligned16(row_codes) || row_ld % 16 || row_ld < cols || !on(row_scales, 4))) return OZK_ERR_INVALID_ARG;
  if (by_cols && (!col_codes || !col_scales || !aligned16(col_codes) || col_ld % 16 || col_ld < cols)) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const Layout l = row_layout(cols, kNormOne);
  const int xs = type_size(x_type), hs = type_size(h_type);
  NormParams p = {};
  p.x = X, p.r = R, p.w = weight, p.h = H, p.y = Y;
  p.ldx = ldx, p.ldr = ldr, p.ldh = ldh, p.ldy = ldy, p.ldq = row_ld;
  p.rows = (int)rows, p.cols = (int)cols, p.w_bf16 = w_type == OZK_BF16, p.warps = l.warps, p.side_rows = l.rows;
  p.eps = (float)eps, p.root = root, p.codes = row_codes, p.scales = reinterpret_cast<uint32_t*>(row_scales);
  const bool vec = quads(X, ldx, xs) && (!R || (quads(R, ldr, hs) && quads(H, ldh, hs))) && (!Y || quads(Y, ldy, xs)) && quads(weight, 0, type_size(w_type));
  if (x_type == OZK_BF16) {
    if (!R) launch_norm_rows<__nv_bfloat16, None>(vec, p, l, st);
    else if (r_type == OZK_BF16) launch_norm_rows<__nv_bfloat16, __nv_bfloat16>(vec, p, l, st);
    else launch_norm_rows<__nv_bfloat16, float>(vec, p, l, st);
  } else {
    if (!R) launch_norm_rows<float, None>(vec, p, l, st);
    else launch_norm_rows<float, float>(vec, p, l, st);
  }
  if (cudaGetLastError() != cudaSuccess) return OZK_ERR_CUDA;
  if (by_cols) {
    const void* h = R ? H : X;
    const int64_t ld = R ? ldh : ldx;
    if (h_type == OZK_BF16) launch_norm_cols<__nv_bfloat16>(quads(h, ld, 2) && quads(weight, 0, type_size(w_type)), h, ld, p, col_codes, col_ld, col_scales, st);
    else launch_norm_cols<float>(quads(h, ld, 4) && quads(weight, 0, type_size(w_type)), h, ld, p, col_codes, col_ld, col_scales, st);
    if (cudaGetLastError() != cudaSuccess) return OZK_ERR_CUDA;
  }
  return OZK_OK;
}

size_t ozk_rms_norm_backward_scratch_bytes(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || cols > kMostCols) return 0;
  const Layout l = row_layout(cols, kGradOne);
  return (size_t)grad_grid(rows, l) * l.rows * (size_t)cols * 4;
}

ozk_status ozk_rms_norm_backward(int64_t rows, int64_t cols, const void* dY, int dy_type, int64_t lddy, const void* H, int h_type, int64_t ldh, const float* root,
                                 const void* weight, int w_type, const void* dH, int64_t lddh, void* dX, int64_t lddx, float* dweight, void* scratch,
                                 size_t scratch_bytes, void* stream) {
  if (rows < 0 || cols < 0 || !type_ok(dy_type) || !type_ok(h_type) || !type_ok(w_type) || lddy < cols || ldh < cols || lddx < cols) return OZK_ERR_INVALID_ARG;
  if (dH && lddh < cols) return OZK_ERR_INVALID_ARG;
  if (rows > INT32_MAX - 1024 || cols > kMostCols) return OZK_ERR_UNSUPPORTED;
  if (cols == 0) return OZK_OK;
  if (dweight && !on(dweight, 4)) return OZK_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) return !dweight || cudaMemsetAsync(dweight, 0, (size_t)cols * 4, st) == cudaSuccess ? OZK_OK : OZK_ERR_CUDA;
  const int ds = type_size(dy_type), hs = type_size(h_type);
  if (!on(dY, ds) || !on(H, hs) || !on(root, 4) || !on(weight, type_size(w_type)) || !on(dX, hs) || (dH && !on(dH, hs))) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  const Layout l = row_layout(cols, kGradOne);
  const int grid = grad_grid(rows, l);
  if (dweight && (!on(scratch, 16) || scratch_bytes < ozk_rms_norm_backward_scratch_bytes(rows, cols))) return OZK_ERR_WORKSPACE;
  GradParams p = {};
  p.dy = dY, p.h = H, p.dh = dH, p.w = weight, p.dx = dX, p.root = root;
  p.lddy = lddy, p.ldh = ldh, p.lddh = lddh, p.lddx = lddx;
  p.rows = (int)rows, p.cols = (int)cols, p.w_bf16 = w_type == OZK_BF16, p.warps = l.warps, p.side_rows = l.rows;
  p.parts = dweight ? static_cast<float*>(scratch) : nullptr;
  const bool vec = quads(dY, lddy, ds) && quads(H, ldh, hs) && quads(dX, lddx, hs) && (!dH || quads(dH, lddh, hs)) && quads(weight, 0, type_size(w_type));
  if (dy_type == OZK_BF16) {
    if (h_type == OZK_BF16) launch_backward<__nv_bfloat16, __nv_bfloat16>(vec, p, l, grid, st);
    else launch_backward<__nv_bfloat16, float>(vec, p, l, grid, st);
  } else {
    if (h_type == OZK_BF16) launch_backward<float, __nv_bfloat16>(vec, p, l, grid, st);
    else launch_backward<float, float>(vec, p, l, grid, st);
  }
  if (cudaGetLastError() != cudaSuccess) return OZK_ERR_CUDA;
  if (dweight) {
    const int64_t parts = rows < (int64_t)grid * l.rows ? rows : (int64_t)grid * l.rows;
    norm_dw_kernel<<<(unsigned)ceil_div(cols, 32), 1024, 0, st>>>(p.parts, (int)parts, p.cols, dweight);
    if (cudaGetLastError() != cudaSuccess) return OZK_ERR_CUDA;
  }
  return OZK_OK;
}

}  // extern "C"
