// The gradients of the RMS norm: g = dy w;  dx = dh + s (g - h s mean(g h s));  dw = sum over the rows of dy h s, in FP32.
// Rows lie over warps as in the forward pass.  Bound by memory and by what a row's sum holds up: 16384 x 4096 BF16 110 us (4.9 TB/s), 8192 x 8192 FP32 200 us (5.4),
// 733 x 16384 FP32 with BF16 dy 50 us (3.4: one thread block a multiprocessor, whose rows have room for one more on its way), 8191 x 4097 BF16 190 us (instructions).
#include "ozk_norm.cuh"

namespace ozk {
namespace {

struct GradParams {
  const void *dy, *h, *dh, *w;
  void* dx;
  const float* root;
  int64_t lddy, ldh, lddh, lddx;
  int rows, cols, w_kind, warps, side_rows;
  float inv_cols;
  float* parts;   // [grid x side_rows][cols], or NULL
};

template <class TD, class TH, int kL, int kE, int V, int kThreads, bool kWhole>
struct GradShape {
  static constexpr int kBlocks = kThreads == 512 ? 1 : V == 1 && sizeof(TD) + sizeof(TH) == 4 ? 3 : 2;
  template <bool kOn>
  static constexpr int bytes() { return Stream<TD, kL, kE, V, kWhole, kOn>::kThread + 2 * Stream<TH, kL, kE, V, kWhole, kOn>::kThread; }
  static constexpr int kStages = ring_stages(bytes<true>(), kThreads, kBlocks);
  static constexpr bool kOn = kStages > 0;
  static constexpr int kThreadBytes = bytes<kOn>();
  // Room for one row only: dy and h stay in registers, so that the next row's may follow before this one's sum is known.
  static constexpr bool kHold = kStages == 1 && V <= 2 && kE > 1;
};

// Rows as in the forward pass; what is needed again after the sum is read again from shared memory.  Each thread adds up its
// columns' share of dw over the rows it sees; norm_dw_kernel adds the thread blocks' sums.
template <class TD, class TH, int kL, int kE, int V, int kThreads, bool kWhole>
__global__ void __launch_bounds__(kThreads, GradShape<TD, TH, kL, kE, V, kThreads, kWhole>::kBlocks) norm_backward_kernel(const __grid_constant__ GradParams p) {
  using S = GradShape<TD, TH, kL, kE, V, kThreads, kWhole>;
  using SD = Stream<TD, kL, kE, V, kWhole, S::kOn>;
  using SH = Stream<TH, kL, kE, V, kWhole, S::kOn>;
  constexpr int kSlots = S::kOn ? S::kStages : 1, kPieces = 16 / kL;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float part[2][kMostWarps];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, in_row = warp % p.warps, step = p.warps * kGroup;
  const int c_warp = in_row * kGroup, c_lane = c_warp + lane * kL, group_left = p.cols - c_warp;
  const int first = (int)blockIdx.x * p.side_rows + warp / p.warps, stride = (int)gridDim.x * p.side_rows;
  const uint32_t slot_bytes = S::kThreadBytes * blockDim.x, h_at = SD::kThread * blockDim.x, e_at = h_at + SH::kThread * blockDim.x, ring_at = smem_u32(ring);
  int row = first, ahead = first;   // the row at hand, and the next to be fetched
  const int64_t d_step = stride * p.lddy, h_step = stride * p.ldh, e_step = stride * p.lddh, o_step = stride * p.lddx;
  const TD *pd = static_cast<const TD*>(p.dy) + row * p.lddy + c_lane, *d_ahead = pd;
  const TH *ph = static_cast<const TH*>(p.h) + row * p.ldh + c_lane, *h_ahead = ph, *pe = p.dh ? static_cast<const TH*>(p.dh) + row * p.lddh + c_lane : nullptr, *e_ahead = pe;
  TH* po = static_cast<TH*>(p.dx) + row * p.lddx + c_lane;
  auto fetch = [&](int slot) {
    if constexpr (S::kOn) {
      if (ahead < p.rows) {
        const bool edge = ahead == 0 || ahead == p.rows - 1;
        SD::fetch(d_ahead, ring_at + slot * slot_bytes, step, lane, group_left, edge);
        SH::fetch(h_ahead, ring_at + slot * slot_bytes + h_at, step, lane, group_left, edge);
        if (pe) SH::fetch(e_ahead, ring_at + slot * slot_bytes + e_at, step, lane, group_left, edge);
      }
      copy_commit();
      ahead += stride, d_ahead += d_step, h_ahead += h_step;
      if (pe) e_ahead += e_step;
    }
  };
  // With one slot: dy and h of the next row once this one's are in registers, dh after it has been written.
  auto fetch_early = [&]() {
    if (ahead < p.rows) {
      const bool edge = ahead == 0 || ahead == p.rows - 1;
      SD::fetch(d_ahead, ring_at, step, lane, group_left, edge);
      SH::fetch(h_ahead, ring_at + h_at, step, lane, group_left, edge);
    }
    d_ahead += d_step, h_ahead += h_step;
  };
  auto fetch_late = [&]() {
    if (pe && ahead < p.rows) SH::fetch(e_ahead, ring_at + e_at, step, lane, group_left, ahead == 0 || ahead == p.rows - 1);
    if (pe) e_ahead += e_step;
    copy_commit();
    ahead += stride;
  };
  if constexpr (S::kHold) {
    fetch_early();
    fetch_late();
  } else {
#pragma unroll
    for (int k = 0; k < kSlots; ++k) fetch(k);
  }
  Piece<TD, kL> d_held[S::kHold ? V : 1][kPieces];
  Piece<TH, kL> h_held[S::kHold ? V : 1][kPieces];
  float dw[V][kPieces][kL];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
      for (int i = 0; i < kL; ++i) dw[v][k][i] = 0.f;
  const int rounds = (p.rows - (int)blockIdx.x * p.side_rows + stride - 1) / stride;   // the same for all threads: they meet at barriers
  int slot = 0;
  float s = row < p.rows ? p.root[row] : 0.f;
  for (int n = 0; n < rounds; ++n) {
    const bool live = row < p.rows, edge = row == 0 || row == p.rows - 1;
    const float s_next = row + stride < p.rows ? p.root[row + stride] : 0.f;
    const uint32_t base = ring_at + slot * slot_bytes;
    float sum = 0.f;
    // Group v of the row, before the sum is known (adds to dw and to the sum) and after (writes dx).
    auto look = [&](auto full, int v, int left) {
      constexpr bool kFull = decltype(full)::value;
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int at = v * step + k * 32 * kL, rest = left - k * 32 * kL;
        Piece<TD, kL> d_now, &d = S::kHold ? d_held[S::kHold ? v : 0][k] : d_now;
        Piece<TH, kL> h_now, &h = S::kHold ? h_held[S::kHold ? v : 0][k] : h_now;
        SD::template take<kFull>(pd, base, at, rest, edge, v, k, d);
        SH::template take<kFull>(ph, base + h_at, at, rest, edge, v, k, h);
        float w[kL];
        load_weights<kFull, kL>(p.w, p.w_kind, c_lane + at, rest, w);
#pragma unroll
        for (int i = 0; i < kL; ++i) {
          const float hn = value(h, i) * s;
          dw[v][k][i] = fmaf(value(d, i), hn, dw[v][k][i]);
          sum = fmaf(value(d, i) * w[i], hn, sum);
        }
      }
    };
    auto write = [&](auto full, int v, int left, float minus_mean) {
      constexpr bool kFull = decltype(full)::value;
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int at = v * step + k * 32 * kL, rest = left - k * 32 * kL;
        Piece<TD, kL> d;
        Piece<TH, kL> h, e = {}, out;
        if constexpr (S::kHold) {
          d = d_held[v][k], h = h_held[v][k];
        } else {
          SD::template take<kFull>(pd, base, at, rest, edge, v, k, d);
          SH::template take<kFull>(ph, base + h_at, at, rest, edge, v, k, h);
        }
        if (pe) SH::template take<kFull>(pe, base + e_at, at, rest, edge, v, k, e);
        float w[kL], dx[kL];
        load_weights<kFull, kL>(p.w, p.w_kind, c_lane + at, rest, w);
#pragma unroll
        for (int i = 0; i < kL; ++i) dx[i] = fmaf(s, fmaf(value(h, i) * s, minus_mean, value(d, i) * w[i]), value(e, i));
#pragma unroll
        for (int i = 0; i < kL; i += 2) set2(out, i, dx[i], dx[i + 1]);
        store_piece<kFull, kE>(po + at, rest, out);
      }
    };
    if constexpr (S::kOn) copy_wait<kSlots - 1>();
    if (live) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int left = group_left - v * step;
        if (left <= 0) continue;
        if constexpr (kWhole) look(std::true_type{}, v, left - lane * kL);
        else if (left >= kGroup) look(std::true_type{}, v, left - lane * kL);
        else look(std::false_type{}, v, left - lane * kL);
      }
    }
    if constexpr (S::kHold) fetch_early();
    sum = row_sum(sum, part, n & 1, p.warps, warp);
    if (live) {
      const float minus_mean = -sum * p.inv_cols;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int left = group_left - v * step;
        if (left <= 0) continue;
        if constexpr (kWhole) write(std::true_type{}, v, left - lane * kL, minus_mean);
        else if (left >= kGroup) write(std::true_type{}, v, left - lane * kL, minus_mean);
        else write(std::false_type{}, v, left - lane * kL, minus_mean);
      }
    }
    if constexpr (S::kHold) {
      fetch_late();
    } else {
      fetch(slot);
      slot = slot + 1 == kSlots ? 0 : slot + 1;
    }
    s = s_next;
    row += stride, pd += d_step, ph += h_step, po += o_step;
    if (pe) pe += e_step;
  }
  if (!p.parts) return;
  float* mine = p.parts + (int64_t)first * p.cols;   // the first row that this warp saw names its sums
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
      for (int i = 0; i < kL; ++i) {
        const int c = c_lane + v * step + k * 32 * kL + i;
        if (c < p.cols) mine[c] = dw[v][k][i];
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
constexpr int kGradBlocks = 3;   // a multiprocessor, at most: what the scratch of the partial sums is for
template <class TD, class TH, int kL, int kE, int V, int kThreads, bool kWhole>
bool launch_backward_as(const GradParams& p, const Layout& l, int* grid, cudaStream_t st) {
  using S = GradShape<TD, TH, kL, kE, V, kThreads, kWhole>;
  static_assert(S::kBlocks <= kGradBlocks, "room for partial sums");
  static std::atomic<bool> done[kMaxDevices];
  auto kernel = norm_backward_kernel<TD, TH, kL, kE, V, kThreads, kWhole>;
  if (!raise_smem(kernel, (size_t)S::kStages * S::kThreadBytes * kThreads, done)) return false;
  const unsigned threads = (unsigned)(32 * l.warps * l.rows);
  *grid = grid_of(p.rows, l, S::kBlocks);
  kernel<<<(unsigned)*grid, threads, (size_t)S::kStages * S::kThreadBytes * threads, st>>>(p);
  return cudaGetLastError() == cudaSuccess;
}
template <class TD, class TH, int kL, int kE, bool kWhole>
bool launch_backward(const GradParams& p, const Layout& l, int* grid, cudaStream_t st) {
  if (l.warps <= 8) return l.v == 1 ? launch_backward_as<TD, TH, kL, kE, 1, 256, kWhole>(p, l, grid, st) : launch_backward_as<TD, TH, kL, kE, 2, 256, kWhole>(p, l, grid, st);
  return l.v == 2 ? launch_backward_as<TD, TH, kL, kE, 2, 512, kWhole>(p, l, grid, st) : launch_backward_as<TD, TH, kL, kE, 4, 512, kWhole>(p, l, grid, st);
}
template <class TD, class TH>
bool launch_backward(int e, const GradParams& p, const Layout& l, int* grid, cudaStream_t st) {
  if constexpr (kAllBf16<TD, TH>) {
    if (e == 8) return p.cols % kGroup == 0 ? launch_backward<TD, TH, 8, 8, true>(p, l, grid, st) : launch_backward<TD, TH, 8, 8, false>(p, l, grid, st);
  } else {
    if (e >= 4 && p.cols % kGroup == 0) return launch_backward<TD, TH, 4, 4, true>(p, l, grid, st);
  }
  return e >= 4 ? launch_backward<TD, TH, 4, 4, false>(p, l, grid, st) : launch_backward<TD, TH, 4, 1, false>(p, l, grid, st);
}

}  // namespace
}  // namespace ozk

using namespace ozk;

extern "C" {

size_t ozk_rms_norm_backward_scratch_bytes(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || cols > kMostCols) return 0;
  const Layout l = row_layout(rows, cols, kGradMost, false);
  return (size_t)grid_of(rows, l, kGradBlocks) * l.rows * (size_t)cols * 4;
}

ozk_status ozk_rms_norm_backward(const ozk_rms_norm_backward_args* args, void* stream) {
  if (!args) return OZK_ERR_INVALID_ARG;
  const ozk_rms_norm_backward_args& a = *args;
  const int64_t rows = a.rows, cols = a.cols;
  if (rows < 0 || cols < 0 || !type_ok(a.dy_type) || !type_ok(a.total_type) || !type_ok(a.weight_type) || a.lddy < cols || a.ldt < cols || a.lddx < cols) return OZK_ERR_INVALID_ARG;
  if (a.dtotal && a.lddt < cols) return OZK_ERR_INVALID_ARG;
  if (rows > kMostRows || cols > kMostCols) return OZK_ERR_UNSUPPORTED;
  if (cols == 0) return OZK_OK;
  if (a.dweight && !on(a.dweight, 4)) return OZK_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) return !a.dweight || cudaMemsetAsync(a.dweight, 0, (size_t)cols * 4, st) == cudaSuccess ? OZK_OK : OZK_ERR_CUDA;
  const int ds = type_size(a.dy_type), hs = type_size(a.total_type);
  if (!on(a.dy, ds) || !on(a.total, hs) || !on(a.root, 4) || !on(a.weight, type_size(a.weight_type)) || !on(a.dx, hs) || (a.dtotal && !on(a.dtotal, hs))) return OZK_ERR_INVALID_ARG;
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  const Layout l = row_layout(rows, cols, kGradMost, false);
  if (a.dweight && (!on(a.scratch, 16) || a.scratch_bytes < ozk_rms_norm_backward_scratch_bytes(rows, cols))) return OZK_ERR_WORKSPACE;
  GradParams p = {};
  p.dy = a.dy, p.h = a.total, p.dh = a.dtotal, p.w = a.weight, p.dx = a.dx, p.root = a.root;
  p.lddy = a.lddy, p.ldh = a.ldt, p.lddh = a.lddt, p.lddx = a.lddx;
  p.rows = (int)rows, p.cols = (int)cols, p.w_kind = weight_kind(a.weight, a.weight_type), p.warps = l.warps, p.side_rows = l.rows;
  p.inv_cols = 1.f / (float)cols;
  p.parts = a.dweight ? static_cast<float*>(a.scratch) : nullptr;
  const int64_t more = rows > 1;
  int vec = least(least(together(a.dy, more * a.lddy, ds), together(a.total, more * a.ldt, hs)), together(a.dx, more * a.lddx, hs));
  if (a.dtotal) vec = least(vec, together(a.dtotal, more * a.lddt, hs));
  int grid = 0;
  bool ok;
  if (a.dy_type == OZK_BF16)
    ok = a.total_type == OZK_BF16 ? launch_backward<__nv_bfloat16, __nv_bfloat16>(vec, p, l, &grid, st) : launch_backward<__nv_bfloat16, float>(vec, p, l, &grid, st);
  else
    ok = a.total_type == OZK_BF16 ? launch_backward<float, __nv_bfloat16>(vec, p, l, &grid, st) : launch_backward<float, float>(vec, p, l, &grid, st);
  if (!ok) return OZK_ERR_CUDA;
  if (a.dweight) {
    const int64_t parts = rows < (int64_t)grid * l.rows ? rows : (int64_t)grid * l.rows;
    norm_dw_kernel<<<(unsigned)ceil_div(cols, 32), 1024, 0, st>>>(p.parts, (int)parts, p.cols, a.dweight);
    if (cudaGetLastError() != cudaSuccess) return OZK_ERR_CUDA;
  }
  return OZK_OK;
}

}  // extern "C"
