// RMS norm with the residual's addition, its answer in E4M3 by blocks of 128, and its gradients.
//
//   h = round(x + r) in the type of r;  s = 1 / sqrt(mean(h^2) + eps);  y = h s w;  codes and scales of y as the quantiser's.
//   g = dy w;  dx = dh + s (g - h s mean(g h s));  dw = sum over the rows of dy h s.
// The norm is of h as it is stored, so that the backward pass, which reads h and s, differentiates what was computed.  Sums and all
// arithmetic in FP32, in an order that follows from sizes, types, alignment (which columns a lane holds) and the number of multiprocessors; y is rounded once, to its codes.
//
// Rows: a row lies over 1 to 16 warps, 512 columns (one word of scales) a warp and step.  A lane holds eight consecutive columns of each 256, or four of
// each 128, so that 16 or 32 lanes hold a block.  Thread blocks stay and take row after row, the next ones already on their way to shared memory.
// Columns: blocks run along the rows, so a second kernel reads h again, tile by tile, with s known.
//
// Bound by memory where rows are long and aligned, and by instructions (about 20 an element) where they are read in words: 16384 x 4096 BF16 with a BF16 stream 82 us
// by rows (5.7 TB/s), 125 us both ways; 4096 x 16384 FP32 144 us (6.1); 5003 x 4100 BF16 with an FP32 stream both ways 84 us; 8191 x 4097 BF16 by rows 109 us
// (2.2 TB/s).  One row of 4096: 3.4 us on the GPU, 9 with the call.
#include "ozk_norm.cuh"

namespace ozk {
namespace {

// ---- scales -----------------------------------------------------------------------------
// Largest magnitude; NaN where one is not a number, whose bits are above all others'.
__device__ __forceinline__ float largest(float m, float x, float y) {
  asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(x)), "f"(fabsf(y)));
  return m;
}
// Maxima are compared as the upper 16 bits of magnitudes, rounded up, two at a time.  That loses nothing: 448 times a power of two has no lower bits, and
// neither a carry into the exponent nor one across 1.75 changes the scale.  What is not finite, or rounds up to infinity, shows as 0x7F80 and more.
constexpr uint32_t kNotFinite = 0x7F80u;
__device__ __forceinline__ uint32_t upper(float m) { return (__float_as_uint(m) + 0xFFFFu) >> 16; }
__device__ __forceinline__ bool not_finite2(uint32_t m) { return (m & 0xFFFFu) >= kNotFinite || m >= kNotFinite << 16; }
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Codes of kL numbers by reciprocals of their scales.  NaN gives NaN; infinities would give 448 and are replaced before.
template <int kL>
__device__ __forceinline__ void codes_of(const float (&y)[kL], const float* recip, int step, uint32_t (&c)[kL / 4]) {
#pragma unroll
  for (int k = 0; k < kL / 4; ++k)
    c[k] = pack4(y[4 * k] * recip[4 * k * step], y[4 * k + 1] * recip[(4 * k + 1) * step], y[4 * k + 2] * recip[(4 * k + 2) * step], y[4 * k + 3] * recip[(4 * k + 3) * step]);
}
__device__ __forceinline__ float finite_or_nan(float y) { return y - (y - y); }   // subtracted, so that a negative zero keeps its sign
template <bool kFull, int kL>
__device__ __forceinline__ void store_codes(uint8_t* p, int left, const uint32_t (&c)[kL / 4]) {
  if (kFull || left >= kL) {
    store_bytes<kL>(p, c);
  } else {
#pragma unroll
    for (int i = 0; i < kL; ++i)
      if (i < left) p[i] = (uint8_t)(c[i / 4] >> (8 * (i % 4)));
  }
}
struct NormParams {
  const void *x, *r, *w;
  void *h, *y;
  int64_t ldx, ldr, ldh, ldy, ldq;
  int rows, cols, w_kind, warps, side_rows;
  float eps, inv_cols;
  float* root;
  uint8_t* codes;
  uint32_t* scales;
};

// 1 / sqrt(sum / cols + eps).  The approximate root is off by two units in its last place: a Newton step with the residual of its product taken exactly
// brings it to the nearest number but for rare cases, and one step does the same for the quotient, so that codes fall where the formula's do.
__device__ __forceinline__ float inverse_root(float sum, float cols, float inv_cols, float eps) {
  float m = sum * inv_cols;
  if (m < 3.0e38f) m = fmaf(fmaf(-m, cols, sum), inv_cols, m);
  m += eps;
  float s = rsqrtf(m);
  if (m > 1.2e-38f && m < 3.0e38f) {
    const float h = m * s, rest = fmaf(m, s, -h);
    s = fmaf(0.5f * s, fmaf(-rest, s, fmaf(-h, s, 1.f)), s);
  }
  return s;
}

struct None {};   // no residual: h is x and is not written
template <class TX, class TR>
struct Stored { using type = TR; };
template <class TX>
struct Stored<TX, None> { using type = TX; };

// h of a lane's elements.  BF16 to BF16: the packed addition rounds the exact sum once, and so does rounding the FP32 sum, which is exact
// wherever it lies near the middle of two BF16 numbers.
template <int kL>
__device__ __forceinline__ void add_piece(const Piece<__nv_bfloat16, kL>& x, Piece<__nv_bfloat16, kL>& h) {
#pragma unroll
  for (int j = 0; j < kL / 2; ++j) {
    const __nv_bfloat162 v = __hadd2_rn(*reinterpret_cast<const __nv_bfloat162*>(&x.w[j]), *reinterpret_cast<const __nv_bfloat162*>(&h.w[j]));
    h.w[j] = *reinterpret_cast<const uint32_t*>(&v);
  }
}
template <class TX, int kL>
__device__ __forceinline__ void add_piece(const Piece<TX, kL>& x, Piece<float, kL>& h) {
#pragma unroll
  for (int i = 0; i < kL; ++i) h.w[i] = __float_as_uint(value(x, i) + __uint_as_float(h.w[i]));
}

// How a kernel of V groups a warp is laid out: thread blocks that share a multiprocessor, rows on their way.
template <class TX, class TR, int kL, int kE, int V, int kThreads, bool kWhole>
struct NormShape {
  static constexpr bool kAdd = !std::is_same<TR, None>::value;
  using TH = typename Stored<TX, TR>::type;
  static constexpr int kPieces = 16 / kL;
  static constexpr int kBlocks = kThreads == 512 ? 1 : V == 4 || (V == 2 && sizeof(TH) == 4) ? 2 : 3;
  template <bool kOn>
  static constexpr int bytes() { return Stream<TX, kL, kE, V, kWhole, kOn>::kThread + (kAdd ? Stream<TH, kL, kE, V, kWhole, kOn>::kThread : 0); }
  static constexpr int kStages = ring_stages(bytes<true>(), kThreads, kBlocks);
  static constexpr bool kOn = kStages > 0;
  static constexpr int kThreadBytes = bytes<kOn>();
};

// One row's share of a warp: h of group v and its sum of squares ...
template <class S, class SX, class SR, bool kFull, class TX, class TH, int kL, int kE>
__device__ __forceinline__ float norm_read(const TX* x, const TH* r, TH* out, uint32_t base, uint32_t r_at, int at, int left, bool edge, int v, Piece<TH, kL> (&h)[16 / kL], float sum) {
#pragma unroll
  for (int k = 0; k < 16 / kL; ++k) {
    const int c = at + k * 32 * kL, rest = left - k * 32 * kL;
    if constexpr (S::kAdd) {
      Piece<TX, kL> q;
      SX::template take<kFull>(x, base, c, rest, edge, v, k, q);
      SR::template take<kFull>(r, base + r_at, c, rest, edge, v, k, h[k]);
      add_piece(q, h[k]);
      store_piece<kFull, kE>(out + c, rest, h[k]);
    } else {
      SX::template take<kFull>(x, base, c, rest, edge, v, k, h[k]);
    }
#pragma unroll
    for (int i = 0; i < kL; ++i) sum = fmaf(value(h[k], i), value(h[k], i), sum);
  }
  return sum;
}
// ... and y of it with its codes; the word of scales for all lanes.  y_out, codes: the lane's first column, or NULL.
template <bool kFull, class TX, class TH, int kL, int kE>
__device__ __forceinline__ uint32_t norm_write(const Piece<TH, kL> (&h)[16 / kL], float s, const void* weights, int w_kind, int c_lane, int left, TX* y_out, uint8_t* codes) {
  constexpr int kPieces = 16 / kL;
  float y[kPieces][kL], top[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int at = k * 32 * kL;
    float w[kL];
    load_weights<kFull, kL>(weights, w_kind, c_lane + at, left - at, w);
    top[k] = 0.f;
#pragma unroll
    for (int i = 0; i < kL; ++i) y[k][i] = value(h[k], i) * s * w[i];
#pragma unroll
    for (int i = 0; i < kL; i += 2) top[k] = largest(top[k], y[k][i], y[k][i + 1]);
    if (y_out) {
      Piece<TX, kL> q;
#pragma unroll
      for (int i = 0; i < kL; i += 2) set2(q, i, y[k][i], y[k][i + 1]);
      store_piece<kFull, kE>(y_out + at, left - at, q);
    }
  }
  if (!codes) return 0u;
  uint32_t tops[kPieces / 2], c[kPieces];
  bool odd = false;
#pragma unroll
  for (int k = 0; k < kPieces / 2; ++k) {
    tops[k] = upper(top[2 * k]) | upper(top[2 * k + 1]) << 16;
#pragma unroll
    for (int d = 1; d < 128 / kL; d *= 2) tops[k] = larger2(tops[k], __shfl_xor_sync(0xFFFFFFFFu, tops[k], d));
    odd = odd || not_finite2(tops[k]);
    c[2 * k] = scale_code(tops[k] << 16), c[2 * k + 1] = scale_code(tops[k] & 0xFFFF0000u);
  }
  const bool bad = __any_sync(0xFFFFFFFFu, odd);
  if (bad) {
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      uint32_t t = 0;
#pragma unroll
      for (int i = 0; i < kL; ++i) t = max(t, finite_bits(y[k][i])), y[k][i] = finite_or_nan(y[k][i]);
#pragma unroll
      for (int d = 1; d < 128 / kL; d *= 2) t = max(t, __shfl_xor_sync(0xFFFFFFFFu, t, d));
      c[k] = scale_code(t);
    }
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    const int at = k * 32 * kL;
    const float recip = scale_recip(c[k]);
    uint32_t q[kL / 4];
    codes_of<kL>(y[k], &recip, 0, q);
    if (kFull || left > at) store_codes<kFull, kL>(codes + at, left - at, q);
  }
  if constexpr (kL == 4) return c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
  const uint32_t mine = c[0] | c[1] << 16;   // lanes 0 .. 15 have blocks 0 and 2, the others blocks 1 and 3
  return mine | __shfl_down_sync(0xFFFFFFFFu, mine, 16) << 8;
}

// kWhole: all groups are full.
template <class TX, class TR, int kL, int kE, int V, int kThreads, bool kWhole>
__global__ void __launch_bounds__(kThreads, NormShape<TX, TR, kL, kE, V, kThreads, kWhole>::kBlocks) norm_rows_kernel(const __grid_constant__ NormParams p) {
  using S = NormShape<TX, TR, kL, kE, V, kThreads, kWhole>;
  using TH = typename S::TH;
  using SX = Stream<TX, kL, kE, V, kWhole, S::kOn>;
  using SR = Stream<TH, kL, kE, V, kWhole, S::kOn>;
  constexpr int kSlots = S::kOn ? S::kStages : 1;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float part[2][kMostWarps];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, in_row = warp % p.warps, step = p.warps * kGroup;
  const int c_warp = in_row * kGroup, c_lane = c_warp + lane * kL, group_left = p.cols - c_warp;   // group v is v * step further
  const uint32_t slot_bytes = S::kThreadBytes * blockDim.x, r_at = SX::kThread * blockDim.x, ring_at = smem_u32(ring);
  int row = (int)blockIdx.x * p.side_rows + warp / p.warps, ahead = row;   // of the row at hand, and of the next to be fetched
  const int stride = (int)gridDim.x * p.side_rows;
  const int64_t x_step = stride * p.ldx, r_step = stride * p.ldr, h_step = stride * p.ldh, q_step = stride * p.ldq, y_step = stride * p.ldy;
  const TX *x = static_cast<const TX*>(p.x) + row * p.ldx + c_lane, *x_ahead = x;
  const TH *r = static_cast<const TH*>(p.r) + row * p.ldr + c_lane, *r_ahead = r;
  TH* out = static_cast<TH*>(p.h) + row * p.ldh + c_lane;
  TX* y = p.y ? static_cast<TX*>(p.y) + row * p.ldy + c_lane : nullptr;
  uint8_t* codes = p.codes ? p.codes + row * p.ldq + c_lane : nullptr;
  auto fetch = [&](int slot) {
    if constexpr (S::kOn) {
      if (ahead < p.rows) {
        const bool edge = ahead == 0 || ahead == p.rows - 1;
        SX::fetch(x_ahead, ring_at + slot * slot_bytes, step, lane, group_left, edge);
        if constexpr (S::kAdd) SR::fetch(r_ahead, ring_at + slot * slot_bytes + r_at, step, lane, group_left, edge);
      }
      copy_commit();
      ahead += stride, x_ahead += x_step;
      if constexpr (S::kAdd) r_ahead += r_step;
    }
  };
#pragma unroll
  for (int k = 0; k < kSlots; ++k) fetch(k);
  const int rounds = (p.rows - (int)blockIdx.x * p.side_rows + stride - 1) / stride;   // the same for all threads: they meet at barriers
  int slot = 0;
  for (int n = 0; n < rounds; ++n) {
    const bool live = row < p.rows, edge = row == 0 || row == p.rows - 1;
    Piece<TH, kL> h[V][16 / kL];
    float sum = 0.f;
    const uint32_t base = ring_at + slot * slot_bytes;
    if constexpr (S::kOn) copy_wait<kSlots - 1>();
    if (live) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int left = group_left - v * step;   // the same for all lanes
        if (left <= 0) continue;
        if (kWhole || left >= kGroup) sum = norm_read<S, SX, SR, true, TX, TH, kL, kE>(x, r, out, base, r_at, v * step, left - lane * kL, edge, v, h[v], sum);
        else if constexpr (!kWhole) sum = norm_read<S, SX, SR, false, TX, TH, kL, kE>(x, r, out, base, r_at, v * step, left - lane * kL, edge, v, h[v], sum);
      }
    }
    fetch(slot);
    slot = slot + 1 == kSlots ? 0 : slot + 1;
    sum = row_sum(sum, part, n & 1, p.warps, warp);
    if (live) {
      const float s = inverse_root(sum, (float)p.cols, p.inv_cols, p.eps);
      if (in_row == 0 && lane == 0 && p.root) p.root[row] = s;
      if (codes || y) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int left = group_left - v * step, at = v * step;
          if (left <= 0) break;
          TX* y_at = y ? y + at : nullptr;
          uint8_t* codes_at = codes ? codes + at : nullptr;
          const uint32_t word = kWhole || left >= kGroup ? norm_write<true, TX, TH, kL, kE>(h[v], s, p.w, p.w_kind, c_lane + at, left - lane * kL, y_at, codes_at)
                                               : norm_write<false, TX, TH, kL, kE>(h[v], s, p.w, p.w_kind, c_lane + at, left - lane * kL, y_at, codes_at);
          if (codes && lane == 0) p.scales[(int64_t)((c_warp + at) / kGroup) * p.rows + row] = word;
        }
      }
    }
    row += stride, x += x_step;
    if constexpr (S::kAdd) r += r_step, out += h_step;
    if (y) y += y_step;
    if (codes) codes += q_step;
  }
}

// Codes by columns: a 128 x 128 tile of h a thread block.  128 / kL lanes hold a row's columns; a thread's rows are kRows apart.
template <class TH, int kL, int kE, bool kFull>
__device__ __forceinline__ void norm_cols_tile(const TH* H, int64_t ldh, const float* root, const void* W, int w_kind, int rows, int cols, uint8_t* Q, int64_t ldq, uint8_t* S,
                                               uint32_t (*part)[kBlock / 2], float* recips, float* roots, int tr, int tc, int tiles_r) {
  constexpr int kLanes = kBlock / kL, kRows = 256 / kLanes, kN = kBlock / kRows;   // lanes a row, rows side by side, rows a thread
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, c_in = threadIdx.x % kLanes * kL, r_in = threadIdx.x / kLanes;
  const int r0 = tr * kBlock, c = tc * kBlock + c_in, left = cols - c;
  Piece<TH, kL> h[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const TH* at = H + (int64_t)(r0 + r_in + kRows * i) * ldh + c;
    const int r = r0 + r_in + kRows * i;
    load_piece<kFull, kE>(at, kFull ? kL : r < rows ? left : 0, r == 0 || r == rows - 1, h[i]);
  }
  if (threadIdx.x < kBlock) roots[threadIdx.x] = kFull || r0 + (int)threadIdx.x < rows ? root[r0 + threadIdx.x] : 0.f;
  float w[kL];
  load_weights<kFull, kL>(W, w_kind, c, left, w);
  __syncthreads();
  float top[kL] = {};
#pragma unroll
  for (int i = 0; i < kN; i += 2) {
    const float s = roots[r_in + kRows * i], t = roots[r_in + kRows * (i + 1)];
#pragma unroll
    for (int j = 0; j < kL; ++j) top[j] = largest(top[j], value(h[i], j) * s * w[j], value(h[i + 1], j) * t * w[j]);
  }
  uint32_t tops[kL / 2], worst = 0;
#pragma unroll
  for (int j = 0; j < kL / 2; ++j) {
    tops[j] = upper(top[2 * j]) | upper(top[2 * j + 1]) << 16;
    worst = larger2(worst, tops[j]);
  }
  const bool bad = __syncthreads_or(not_finite2(worst));
  if (bad) {   // again without them; magnitudes that round up to infinity count as the largest below it, which has the same scale
#pragma unroll
    for (int j = 0; j < kL / 2; ++j) {
      uint32_t a = 0, b = 0;
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const float s = roots[r_in + kRows * i];
        a = max(a, finite_bits(value(h[i], 2 * j) * s * w[2 * j])), b = max(b, finite_bits(value(h[i], 2 * j + 1) * s * w[2 * j + 1]));
      }
      tops[j] = min(upper(__uint_as_float(a)), kNotFinite - 1) | min(upper(__uint_as_float(b)), kNotFinite - 1) << 16;
    }
  }
  if constexpr (kLanes == 16) {
#pragma unroll
    for (int j = 0; j < kL / 2; ++j) tops[j] = larger2(tops[j], __shfl_xor_sync(0xFFFFFFFFu, tops[j], 16));
  }
  if (lane < kLanes) store_bytes<2 * kL>(&part[warp][c_in / 2], tops);
  __syncthreads();
  if (threadIdx.x < kBlock) {
    uint32_t t = part[0][threadIdx.x / 2];
#pragma unroll
    for (int i = 1; i < 8; ++i) t = larger2(t, part[i][threadIdx.x / 2]);
    const uint32_t code = scale_code(threadIdx.x % 2 ? t & 0xFFFF0000u : t << 16);
    recips[threadIdx.x] = scale_recip(code);
    const int col = tc * kBlock + (int)threadIdx.x;
    if (col < cols) {
      uint8_t* s = S + ((int64_t)(tr / 4) * cols + col) * 4;
      s[tr % 4] = (uint8_t)code;
      if (tr + 1 == tiles_r)
        for (int b = tr % 4 + 1; b < 4; ++b) s[b] = 127;
    }
  }
  __syncthreads();
  float recip[kL];
#pragma unroll
  for (int j = 0; j < kL; j += 4) {
    const float4 f = *reinterpret_cast<const float4*>(&recips[c_in + j]);
    recip[j] = f.x, recip[j + 1] = f.y, recip[j + 2] = f.z, recip[j + 3] = f.w;
  }
  auto write = [&](auto odd) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int r = r0 + r_in + kRows * i;
      const float s = roots[r_in + kRows * i];
      float y[kL];
#pragma unroll
      for (int j = 0; j < kL; ++j) {
        y[j] = value(h[i], j) * s * w[j];
        if constexpr (decltype(odd)::value) y[j] = finite_or_nan(y[j]);
      }
      uint32_t q[kL / 4];
      codes_of<kL>(y, recip, 1, q);
      if (kFull || (r < rows && left > 0)) store_codes<kFull, kL>(Q + (int64_t)r * ldq + c, left, q);
    }
  };
  if (bad) write(std::true_type{}); else write(std::false_type{});
}
template <class TH, int kL, int kE>
__global__ void __launch_bounds__(256, sizeof(TH) == 2 ? 3 : 2) norm_cols_kernel(const TH* H, int64_t ldh, const float* root, const void* W, int w_kind, int rows, int cols,
                                                                               uint8_t* Q, int64_t ldq, uint8_t* S) {
  __shared__ __align__(16) uint32_t part[8][kBlock / 2];
  __shared__ __align__(16) float recips[kBlock];
  __shared__ float roots[kBlock];
  const int tiles_c = (cols + kBlock - 1) / kBlock, tiles_r = (rows + kBlock - 1) / kBlock;
  const int tile = (int)(gridDim.x - 1 - blockIdx.x);   // from the end, which the rows' kernel has just written: it is still in L2
  const int tr = tile / tiles_c, tc = tile % tiles_c;
  if (tr * kBlock + kBlock <= rows && tc * kBlock + kBlock <= cols)
    norm_cols_tile<TH, kL, kE, true>(H, ldh, root, W, w_kind, rows, cols, Q, ldq, S, part, recips, roots, tr, tc, tiles_r);
  else
    norm_cols_tile<TH, kL, kE, false>(H, ldh, root, W, w_kind, rows, cols, Q, ldq, S, part, recips, roots, tr, tc, tiles_r);
}

// ---- host side ----------------------------------------------------------------------------
template <class TX, class TR, int kL, int kE, int V, int kThreads, bool kWhole>
bool launch_norm_rows_as(const NormParams& p, const Layout& l, cudaStream_t st) {
  using S = NormShape<TX, TR, kL, kE, V, kThreads, kWhole>;
  static std::atomic<bool> done[kMaxDevices];
  auto kernel = norm_rows_kernel<TX, TR, kL, kE, V, kThreads, kWhole>;
  if (!raise_smem(kernel, (size_t)S::kStages * S::kThreadBytes * kThreads, done)) return false;
  const unsigned threads = (unsigned)(32 * l.warps * l.rows);
  kernel<<<(unsigned)grid_of(p.rows, l, S::kBlocks), threads, (size_t)S::kStages * S::kThreadBytes * threads, st>>>(p);
  return cudaGetLastError() == cudaSuccess;
}
template <class TX, class TR, int kL, int kE, bool kWhole>
bool launch_norm_rows(const NormParams& p, const Layout& l, cudaStream_t st) {
  if (l.warps > 8) {
    if constexpr (sizeof(typename Stored<TX, TR>::type) == 4) {
      if (l.v == 2) return launch_norm_rows_as<TX, TR, kL, kE, 2, 512, kWhole>(p, l, st);
    }
    return launch_norm_rows_as<TX, TR, kL, kE, 4, 512, kWhole>(p, l, st);
  }
  if (l.v == 1) return launch_norm_rows_as<TX, TR, kL, kE, 1, 256, kWhole>(p, l, st);
  if constexpr (sizeof(typename Stored<TX, TR>::type) == 2) {
    if (l.v == 4) return launch_norm_rows_as<TX, TR, kL, kE, 4, 256, kWhole>(p, l, st);
  }
  return launch_norm_rows_as<TX, TR, kL, kE, 2, 256, kWhole>(p, l, st);
}
template <class TX, class TR>
bool launch_norm_rows(int e, const NormParams& p, const Layout& l, cudaStream_t st) {
  if constexpr (kAllBf16<TX, TR>) {
    if (e == 8) return p.cols % kGroup == 0 ? launch_norm_rows<TX, TR, 8, 8, true>(p, l, st) : launch_norm_rows<TX, TR, 8, 8, false>(p, l, st);
  } else {
    if (e >= 4 && p.cols % kGroup == 0) return launch_norm_rows<TX, TR, 4, 4, true>(p, l, st);
  }
  return e >= 4 ? launch_norm_rows<TX, TR, 4, 4, false>(p, l, st) : launch_norm_rows<TX, TR, 4, 1, false>(p, l, st);
}
template <class TH, int kL, int kE>
void launch_norm_cols(const void* h, int64_t ldh, const NormParams& p, uint8_t* q, int64_t ldq, uint8_t* s, cudaStream_t st) {
  const unsigned tiles = (unsigned)(ceil_div(p.rows, kBlock) * ceil_div(p.cols, kBlock));
  norm_cols_kernel<TH, kL, kE><<<tiles, 256, 0, st>>>(static_cast<const TH*>(h), ldh, p.root, p.w, p.w_kind, p.rows, p.cols, q, ldq, s);
}
template <class TH>
void launch_norm_cols(int e, const void* h, int64_t ldh, const NormParams& p, uint8_t* q, int64_t ldq, uint8_t* s, cudaStream_t st) {
  if constexpr (sizeof(TH) == 2) {
    if (e == 8) return launch_norm_cols<TH, 8, 8>(h, ldh, p, q, ldq, s, st);
  }
  if (e >= 4) launch_norm_cols<TH, 4, 4>(h, ldh, p, q, ldq, s, st); else launch_norm_cols<TH, 4, 1>(h, ldh, p, q, ldq, s, st);
}

}  // namespace
}  // namespace ozk

using namespace ozk;

extern "C" {

ozk_status ozk_rms_norm(const ozk_rms_norm_args* args, void* stream) {
  if (!args) return OZK_ERR_INVALID_ARG;
  const ozk_rms_norm_args& a = *args;
  const int64_t rows = a.rows, cols = a.cols;
  const void *X = a.x, *R = a.residual;
  if (rows < 0 || cols < 0 || !type_ok(a.x_type) || !type_ok(a.weight_type) || a.ldx < cols || !(a.eps >= 0.0)) return OZK_ERR_INVALID_ARG;
  if (R && (!type_ok(a.residual_type) || a.ldr < cols || a.ldt < cols)) return OZK_ERR_INVALID_ARG;
  if (rows > kMostRows || cols > kMostCols || (R && a.residual_type != a.x_type && a.residual_type != OZK_F32)) return OZK_ERR_UNSUPPORTED;
  const bool by_rows = a.row_codes || a.row_scales, by_cols = a.col_codes || a.col_scales;
  if (rows == 0 || cols == 0) return OZK_OK;
  const int h_type = R ? a.residual_type : a.x_type, xs = type_size(a.x_type), hs = type_size(h_type);
  if (!on(X, xs) || !on(a.weight, type_size(a.weight_type)) || (R && (!on(R, hs) || !on(a.total, hs)))) return OZK_ERR_INVALID_ARG;
  if (a.y && (!on(a.y, xs) || a.ldy < cols || a.y == (R ? a.total : X))) return OZK_ERR_INVALID_ARG;   // what is normed is read again for the columns
  if ((a.root && !on(a.root, 4)) || (by_cols && !a.root)) return OZK_ERR_INVALID_ARG;
  if (by_rows && (!a.row_codes || !a.row_scales || !aligned16(a.row_codes) || a.row_ld % 16 || a.row_ld < cols || !on(a.row_scales, 4))) return OZK_ERR_INVALID_ARG;
  if (by_cols && (!a.col_codes || !a.col_scales || !aligned16(a.col_codes) || a.col_ld % 16 || a.col_ld < cols)) return OZK_ERR_INVALID_ARG;
  if (by_cols && ceil_div(rows, kBlock) * ceil_div(cols, kBlock) > INT32_MAX) return OZK_ERR_UNSUPPORTED;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const Layout l = row_layout(rows, cols, h_type == OZK_F32 ? kNormMostF32 : kNormMost, true);
  NormParams p = {};
  p.x = X, p.r = R, p.w = a.weight, p.h = a.total, p.y = a.y;
  p.ldx = a.ldx, p.ldr = a.ldr, p.ldh = a.ldt, p.ldy = a.ldy, p.ldq = a.row_ld;
  p.rows = (int)rows, p.cols = (int)cols, p.w_kind = weight_kind(a.weight, a.weight_type), p.warps = l.warps, p.side_rows = l.rows;
  p.eps = (float)a.eps, p.inv_cols = 1.f / (float)cols, p.root = a.root, p.codes = a.row_codes, p.scales = reinterpret_cast<uint32_t*>(a.row_scales);
  const int64_t more = rows > 1;   // a single row's stride does not matter
  int vec = together(X, more * a.ldx, xs);
  if (R) vec = least(vec, least(together(R, more * a.ldr, hs), together(a.total, more * a.ldt, hs)));
  if (a.y) vec = least(vec, together(a.y, more * a.ldy, xs));
  bool ok;
  if (a.x_type == OZK_BF16)
    ok = !R ? launch_norm_rows<__nv_bfloat16, None>(vec, p, l, st)
            : h_type == OZK_BF16 ? launch_norm_rows<__nv_bfloat16, __nv_bfloat16>(vec, p, l, st) : launch_norm_rows<__nv_bfloat16, float>(vec, p, l, st);
  else
    ok = !R ? launch_norm_rows<float, None>(vec, p, l, st) : launch_norm_rows<float, float>(vec, p, l, st);
  if (!ok) return OZK_ERR_CUDA;
  if (by_cols) {
    const void* h = R ? a.total : X;
    const int64_t ld = R ? a.ldt : a.ldx;
    if (h_type == OZK_BF16) launch_norm_cols<__nv_bfloat16>(together(h, more * ld, 2), h, ld, p, a.col_codes, a.col_ld, a.col_scales, st);
    else launch_norm_cols<float>(together(h, more * ld, 4), h, ld, p, a.col_codes, a.col_ld, a.col_scales, st);
    if (cudaGetLastError() != cudaSuccess) return OZK_ERR_CUDA;
  }
  return OZK_OK;
}

}  // extern "C"
