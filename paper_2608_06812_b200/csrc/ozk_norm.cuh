// What the norm and its gradients share: rows in pieces of a lane, rows on their way to shared memory, sums over a row's warps, layouts.
#pragma once

#include <type_traits>

#include "ozk_fp8_product.cuh"

namespace ozk {
namespace {

using namespace fp8;

// ---- consecutive elements of a lane ---------------------------------------------------------
constexpr int kGroup = 512;   // columns a warp holds at a time
template <class T, int kL>
struct Piece {
  uint32_t w[kL * sizeof(T) / 4];
};
template <int kL>
__device__ __forceinline__ float value(const Piece<__nv_bfloat16, kL>& q, int i) { return i % 2 ? bf16_hi(q.w[i / 2]) : bf16_lo(q.w[i / 2]); }
template <int kL>
__device__ __forceinline__ float value(const Piece<float, kL>& q, int i) { return __uint_as_float(q.w[i]); }
// Two elements, rounded to the type.
template <int kL>
__device__ __forceinline__ void set2(Piece<__nv_bfloat16, kL>& q, int i, float a, float b) { q.w[i / 2] = pack_bf16(a, b); }
template <int kL>
__device__ __forceinline__ void set2(Piece<float, kL>& q, int i, float a, float b) { q.w[i] = __float_as_uint(a), q.w[i + 1] = __float_as_uint(b); }

// What is read once need not stay in L1; not through the read-only path, because h may be written over x or r.
template <int kBytes>
__device__ __forceinline__ void load_bytes(const void* p, uint32_t* w) {
  if constexpr (kBytes == 16) asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
  else if constexpr (kBytes == 8) asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
  else if constexpr (kBytes == 4) asm volatile("ld.global.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
}
template <int kBytes>
__device__ __forceinline__ void store_bytes(void* p, const uint32_t* w) {
  if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
}
__device__ __forceinline__ uint32_t load_16(const void* p) {
  uint16_t v;
  asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
  return v;
}
// Bytes of one access: kE elements, as far as places and strides allow, and 16 bytes at most.
template <class T, int kE>
__host__ __device__ constexpr int access() { return kE * (int)sizeof(T) > 16 ? 16 : kE * (int)sizeof(T); }
// BF16 rows at odd places: a lane's elements are cut from the 4-byte words that hold them.  The words at a row's ends hold a neighbour's element too, which
// in the matrix's first and last rows (`edge`) may not be there: these two are read element by element.
template <class T, int kE>
__host__ __device__ constexpr bool odd_places() { return sizeof(T) == 2 && kE == 1; }
__device__ __forceinline__ int at_odd(const void* p) { return (int)(reinterpret_cast<uintptr_t>(p) & 2); }
template <int kWords>
__device__ __forceinline__ void cut(const uint32_t* in, int odd, uint32_t* out) {
#pragma unroll
  for (int i = 0; i < kWords; ++i) out[i] = __funnelshift_r(in[i], in[i + 1], 8 * odd);
}
// The lane's elements from `p` on.  kFull: all belong to the row; otherwise `left` of them do, and the others are zero.
template <bool kFull, int kE, class T, int kL>
__device__ __forceinline__ void load_piece(const T* p, int left, bool edge, Piece<T, kL>& q) {
  constexpr int kBytes = access<T, kE>(), kStep = kBytes / (int)sizeof(T);
  if constexpr (odd_places<T, kE>()) {
    if ((kFull || left >= kL) && !edge) {
      const int odd = at_odd(p);
      const char* from = reinterpret_cast<const char*>(p) - odd;
      uint32_t w[kL / 2 + 1];
#pragma unroll
      for (int i = 0; i < kL / 2; ++i) load_bytes<4>(from + 4 * i, w + i);
      w[kL / 2] = 0;
      if (odd) load_bytes<4>(from + 2 * kL, w + kL / 2);
      cut<kL / 2>(w, odd, q.w);
      return;
    }
  } else if (kFull || left >= kL) {
#pragma unroll
    for (int i = 0; i < kL; i += kStep) load_bytes<kBytes>(p + i, q.w + i * (int)sizeof(T) / 4);
    return;
  }
  if constexpr (!kFull || odd_places<T, kE>()) {
#pragma unroll
    for (int i = 0; i < kL; ++i) {
      if constexpr (sizeof(T) == 2) {
        const uint32_t v = i < left ? load_16(p + i) : 0u;
        q.w[i / 2] = i % 2 ? q.w[i / 2] | v << 16 : v;
      } else {
        q.w[i] = 0u;
        if (i < left) load_bytes<4>(p + i, q.w + i);
      }
    }
  }
}
template <bool kFull, int kE, class T, int kL>
__device__ __forceinline__ void store_piece(T* p, int left, const Piece<T, kL>& q) {
  constexpr int kBytes = access<T, kE>(), kStep = kBytes / (int)sizeof(T);
  if (kFull || left >= kL) {
    if constexpr (!odd_places<T, kE>()) {
#pragma unroll
      for (int i = 0; i < kL; i += kStep) store_bytes<kBytes>(p + i, q.w + i * (int)sizeof(T) / 4);
    } else if (at_odd(p)) {
      reinterpret_cast<uint16_t*>(p)[0] = (uint16_t)q.w[0];
#pragma unroll
      for (int i = 1; i < kL - 1; i += 2) *reinterpret_cast<uint32_t*>(p + i) = __funnelshift_r(q.w[i / 2], q.w[i / 2 + 1], 16);
      reinterpret_cast<uint16_t*>(p)[kL - 1] = (uint16_t)(q.w[kL / 2 - 1] >> 16);
    } else {
#pragma unroll
      for (int i = 0; i < kL; i += 2) store_bytes<4>(p + i, q.w + i / 2);
    }
    return;
  }
  if constexpr (!kFull) {
#pragma unroll
    for (int i = 0; i < kL; ++i) {
      if (i >= left) continue;
      if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(p + i) = (uint16_t)(q.w[i / 2] >> (16 * (i % 2)));
      else store_bytes<4>(p + i, q.w + i);
    }
  }
}
// Weights: cols numbers of either type; a lane's are read together where the array is aligned for it.
enum { kWeightBf16 = 1, kWeightLoose = 2 };
template <bool kFull, int kL>
__device__ __forceinline__ void load_weights(const void* w, int kind, int c, int left, float (&v)[kL]) {
  if ((kFull || left >= kL) && !(kind & kWeightLoose)) {
    if (kind & kWeightBf16) {
      Piece<__nv_bfloat16, kL> q;
      if constexpr (kL == 8) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w) + c));
        q.w[0] = u.x, q.w[1] = u.y, q.w[2] = u.z, q.w[3] = u.w;
      } else {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(w) + c));
        q.w[0] = u.x, q.w[1] = u.y;
      }
#pragma unroll
      for (int i = 0; i < kL; ++i) v[i] = value(q, i);
    } else {
#pragma unroll
      for (int i = 0; i < kL; i += 4) {
        const float4 f = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + c + i));
        v[i] = f.x, v[i + 1] = f.y, v[i + 2] = f.z, v[i + 3] = f.w;
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kL; ++i)
    v[i] = i >= left ? 0.f : kind & kWeightBf16 ? __bfloat162float(__ldg(static_cast<const __nv_bfloat16*>(w) + c + i)) : __ldg(static_cast<const float*>(w) + c + i);
}

// ---- rows on their way ----------------------------------------------------------------------
// A thread copies its own elements of the rows it will see next to shared memory and reads back nobody else's, so that no barrier is needed, no
// register holds what is in flight, and a row's reduction does not hold up the next one's loads.  A lane's elements that the row ends among are read directly.
constexpr int kRingBytes = 200 << 10;   // of a multiprocessor's shared memory
template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }
template <int kBytes>
__device__ __forceinline__ void load_shared(uint32_t at, uint32_t* w) {
  if constexpr (kBytes == 16) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
  else if constexpr (kBytes == 8) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
  else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
}
template <class T, int kL, int kE, int V, bool kWhole, bool kOn>
struct Stream {
  static constexpr bool kOdd = odd_places<T, kE>();
  static constexpr int kBytes = kOdd ? 4 : access<T, kE>(), kStep = kBytes / (int)sizeof(T), kCopies = kL / kStep + (kOdd ? 1 : 0), kPieces = 16 / kL;
  static constexpr int kThread = kOn ? V * kPieces * kCopies * kBytes : 0;   // bytes of a thread's share of a row
  // Copy i of piece k of group v: the threads' copies lie side by side.
  __device__ static __forceinline__ uint32_t place(uint32_t base, int v, int k, int i) { return base + (uint32_t)((((v * kPieces + k) * kCopies + i) * (int)blockDim.x) + (int)threadIdx.x) * kBytes; }
  // row: the lane's first column in the row; group_left: columns of the row from the warp's group on.
  __device__ static __forceinline__ void fetch(const T* row, uint32_t base, int step, int lane, int group_left, bool edge) {
    if constexpr (kOn) {
      const int odd = kOdd ? at_odd(row) : 0;
      if (kOdd && edge) return;
      const char* from = reinterpret_cast<const char*>(row) - odd;
      auto copy = [&](int v, int k) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i)
          if (!kOdd || i + 1 < kCopies || odd) copy_async<kBytes>(place(base, v, k, i), from + (int64_t)(v * step + k * 32 * kL) * (int)sizeof(T) + i * kBytes);
      };
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int left = group_left - v * step;   // the same for all lanes
        if (kWhole ? left > 0 : left >= kGroup) {
#pragma unroll
          for (int k = 0; k < kPieces; ++k) copy(v, k);
        } else if (!kWhole && left > 0) {
#pragma unroll
          for (int k = 0; k < kPieces; ++k)
            if (left - k * 32 * kL - lane * kL >= kL) copy(v, k);
        }
      }
    }
  }
  template <bool kFull>
  __device__ static __forceinline__ void take(const T* row, uint32_t base, int at, int left, bool edge, int v, int k, Piece<T, kL>& out) {
    if constexpr (kOn) {
      if ((kFull || left >= kL) && !(kOdd && edge)) {
        uint32_t w[kCopies * kBytes / 4];
#pragma unroll
        for (int i = 0; i < kCopies; ++i) load_shared<kBytes>(place(base, v, k, i), w + i * kBytes / 4);
        if constexpr (kOdd) {
          cut<kL / 2>(w, at_odd(row), out.w);
        } else {
#pragma unroll
          for (int i = 0; i < kL * (int)sizeof(T) / 4; ++i) out.w[i] = w[i];
        }
        return;
      }
    }
    load_piece<kFull, kE>(row + at, left, edge, out);
  }
};
// Rows that are on their way for each thread block of `threads` that shares a multiprocessor with `blocks - 1` others.
constexpr int ring_stages(int thread_bytes, int threads, int blocks) {
  const int room = thread_bytes ? kRingBytes / blocks / (thread_bytes * threads) : 0;
  return room > 2 ? 2 : room;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

constexpr int kMostWarps = 16;
constexpr int kMostCols = kGroup * kMostWarps * 4;
constexpr int64_t kMostRows = INT32_MAX - 65536;   // row indexes are ints, with room for what lies ahead

// How a row is laid over a thread block: `warps` a row, `rows` of them side by side, V groups of 512 columns a warp.
struct Layout {
  int warps, rows, v;
};
// Forward, a row's own cost (its sum, addresses, barriers) is shared by two groups a warp where there are rows enough to fill the GPU all the same (16384 x 4096: 82 us, one
// group a warp 99); few rows have as many warps as they can use.  The backward pass, whose sums of dw take registers, is faster with one (108 us : 114).  `most`: groups a warp takes in thread blocks of eight warps; wider rows have thread blocks of 16.
Layout row_layout(int64_t rows, int64_t cols, int most, bool forward) {
  const int groups = (int)ceil_div(cols, kGroup);
  int v = forward && groups > 1 && rows * groups >= (int64_t)device_sm_count() * 64 ? 2 : 1;
  while (v < most && 8 * v < groups) v *= 2;
  if (8 * v < groups) v = groups <= 32 ? 2 : 4;
  const int warps = (int)ceil_div(groups, v);
  return {warps, warps < 8 ? 8 / warps : 1, v};
}
constexpr int kNormMost = 4, kNormMostF32 = 2, kGradMost = 2;   // FP32 rows: what four groups hold leaves no room for the next row
// Sum over the warps of this thread's row, the same in all of them.  `side` alternates, so that one barrier is enough.
__device__ __forceinline__ float row_sum(float v, float (*part)[kMostWarps], int side, int warps, int warp) {
  v = warp_sum(v);
  if (warps == 1) return v;
  if (threadIdx.x % 32 == 0) part[side][warp] = v;
  __syncthreads();
  const int i = threadIdx.x % 16;   // both halves of the warp alike
  v = i < warps ? part[side][warp / warps * warps + i] : 0.f;
#pragma unroll
  for (int d = 8; d > 0; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// ---- host side ----------------------------------------------------------------------------
bool type_ok(int t) { return t == OZK_F32 || t == OZK_BF16; }
int type_size(int t) { return t == OZK_F32 ? 4 : 2; }
bool on(const void* p, int size) { return p && (reinterpret_cast<uintptr_t>(p) & (size - 1)) == 0; }
// How many elements a row's place and stride let be read together: 16 bytes at most; 8, 4 or 1.
int together(const void* p, int64_t ld, int size) {
  for (int n = size == 2 ? 8 : 4; n > 2; n /= 2)
    if ((reinterpret_cast<uintptr_t>(p) & (n * size - 1)) == 0 && ld % n == 0) return n;
  return 1;
}
int least(int a, int b) { return a < b ? a : b; }
// Lanes take eight columns where all is BF16 and aligned; FP32 comes in 16-byte accesses of four.
template <class TX, class TR>
constexpr bool kAllBf16 = sizeof(TX) == 2 && !std::is_same<TR, float>::value;

int weight_kind(const void* w, int type) { return (type == OZK_BF16 ? kWeightBf16 : 0) | (aligned16(w) ? 0 : kWeightLoose); }

// Thread blocks of a persistent kernel: what runs at once, or what there is to do.
// `blocks` of them share a multiprocessor where they have 256 or 512 threads, more where they have fewer.
int grid_of(int64_t rows, const Layout& l, int blocks) {
  const int warps = l.warps * l.rows;
  const int64_t need = ceil_div(rows, l.rows), room = (int64_t)device_sm_count() * (warps <= 8 ? blocks * 8 / warps : blocks);
  return (int)(need < room ? need : room);
}

}  // namespace
}  // namespace ozk
