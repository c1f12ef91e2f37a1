// One AdamW step over many tensors in one launch, first and second moments in 32 bits or as E4M3 with a scale per 128.
//
// Every element is read and written once: 16.1 bytes with FP32 parameters, their BF16 copy, BF16 gradients and 8-bit states.  A warp
// works on four blocks of 128 with a block's 128 elements over its lanes, so that a block's maximum is one warp reduction.
// 256 M such parameters: 0.67 ms, 5.9 TB/s (0.75 ms in a long loop of them), bound by memory.  26 M BF16 parameters with 8-bit states (10.1 bytes): 71 us, 3.6 TB/s, bound
// by the arithmetic, most of it the hash, the stochastic roundings and the maxima.  150 tensors of 5000: 6 us, and 7 us a step
// of a loop, which the host needs to launch it.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "ozk_fp8.cuh"

namespace ozk {
namespace {

using namespace fp8;

// A piece is what one warp works on at a time: four blocks of 128 elements.  All its loads are issued before the first result
// is formed (with 8-bit states and FP32 parameters 4 to 5 KiB a warp), which is what keeps enough bytes in flight.
constexpr int kPieceBlocks = 4;
constexpr int kPiece = kPieceBlocks * kBlock;
// Tensors per launch: the table travels in the parameters, which the host copies at every launch, and a launch more costs more than that.
// Up to 192 tensors take the small table, more of them launches of 448 (the most that parameters hold) and a small one for a rest.  A step
// of n tensors of 5000 in a loop, us, small : large tables only: n = 20 5.5 : 6.7, 150 6.3 : 7.3, 200 11.4 : 7.6, 300 12.6 : 10.2, 448 19.5 : 11.5,
// 1000 47 : 33.
constexpr int kFewTensors = 192, kMostTensors = 448;

struct Entry {
  void* param;
  const void* grad;
  void* m;
  void* v;
  uint8_t* m_scale;
  uint8_t* v_scale;
  __nv_bfloat16* copy;
  int64_t n;        // negative: not all arrays are aligned for vector access, -n elements
};
struct Step {
  int count;
  uint32_t first_tensor;              // index in the caller's array of entry 0: part of the hash
  uint32_t pieces;
  const float* grad_scale;
  const int* skip;
  float beta1, one_minus_beta1, beta2, one_minus_beta2, decay, step_size, root_bias, eps;
  uint32_t seed_key;                  // mix(seed)
};
template <int kTensors>
struct Table : Step {
  uint32_t first_piece[kTensors + 1];
  Entry entry[kTensors];
};
static_assert(sizeof(Table<kMostTensors>) <= 32764, "kernel parameters");

// A published hash of 32 bits (Chris Wellons, "Prospecting for Hash Functions", 2018: lowbias32).
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

// mix() of four consecutive numbers a, a ^ 1, a ^ 2, a ^ 3 (the first a multiple of four, XORed with anything): the low two bits do not
// reach the first shift's result, so that step is done once.
__device__ __forceinline__ void mix4(uint32_t a, uint32_t (&out)[4]) {
  const uint32_t t = a ^ (a >> 16);
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    uint32_t x = (t ^ i) * 0x7feb352du;
    x ^= x >> 15;
    x *= 0x846ca68bu;
    out[i] = x ^ (x >> 16);
  }
}

__device__ __forceinline__ Pair multiply_add(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
// Sums one by one: a packed sum of packed products came out as if it had been contracted into multiply-adds (one in 400 moments,
// those whose terms lie at the middle of two codes or cancel, got another code than with both products rounded).
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
  const float2 x = both(a), y = both(b);
  return pair(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y));
}

// Four consecutive elements as they lie in memory, read ahead; `vec`: in one access.  Zeros beyond `left`.
template <class T>
struct Raw;
template <>
struct Raw<float> {
  float4 w;
  __device__ __forceinline__ void load(const float* p, bool vec, int64_t left) {
    if (vec) {
      w = *reinterpret_cast<const float4*>(p);
    } else {
      w.x = left > 0 ? p[0] : 0.f, w.y = left > 1 ? p[1] : 0.f, w.z = left > 2 ? p[2] : 0.f, w.w = left > 3 ? p[3] : 0.f;
    }
  }
  __device__ __forceinline__ Pair lo() const { return pair(w.x, w.y); }
  __device__ __forceinline__ Pair hi() const { return pair(w.z, w.w); }
};
template <>
struct Raw<__nv_bfloat16> {
  uint2 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, bool vec, int64_t left) {
    if (vec) {
      w = *reinterpret_cast<const uint2*>(p);
    } else {
      const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
      w.x = (left > 0 ? q[0] : 0u) | (left > 1 ? (uint32_t)q[1] << 16 : 0u);
      w.y = (left > 2 ? q[2] : 0u) | (left > 3 ? (uint32_t)q[3] << 16 : 0u);
    }
  }
  __device__ __forceinline__ Pair lo() const { return pair(bf16_lo(w.x), bf16_hi(w.x)); }
  __device__ __forceinline__ Pair hi() const { return pair(bf16_lo(w.y), bf16_hi(w.y)); }
};
template <>
struct Raw<uint8_t> {   // E4M3 codes
  uint32_t w;
  __device__ __forceinline__ void load(const uint8_t* p, bool vec, int64_t left) {
    if (vec) {
      w = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w = (left > 0 ? p[0] : 0u) | (left > 1 ? (uint32_t)p[1] << 8 : 0u) | (left > 2 ? (uint32_t)p[2] << 16 : 0u) | (left > 3 ? (uint32_t)p[3] << 24 : 0u);
    }
  }
  __device__ __forceinline__ Pair lo() const {
    const float2 f = unpack2(w & 0xFFFFu);
    return pair(f.x, f.y);
  }
  __device__ __forceinline__ Pair hi() const {
    const float2 f = unpack2(w >> 16);
    return pair(f.x, f.y);
  }
};
__device__ __forceinline__ void store4(float* p, bool vec, int64_t left, const float (&x)[4]) {
  if (vec) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = x[i];
  }
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, bool vec, int64_t left, const float (&x)[4]) {
  if (vec) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = __float2bfloat16_rn(x[i]);
  }
}
__device__ __forceinline__ void store4(uint8_t* p, bool vec, int64_t left, uint32_t w) {
  if (vec) {
    *reinterpret_cast<uint32_t*>(p) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = (uint8_t)(w >> (8 * i));
  }
}

// The root: rounded correctly where it is stored in 8 bits, since a stochastic rounding that falls the other way would be seen in every
// step that follows; to one unit in the last place where only the step is divided by it.  Below FP32's normal range it is zero.
template <bool kExact>
__device__ __forceinline__ float root(float v) {
  float r;
  if constexpr (kExact) asm("sqrt.rn.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); else asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// scale_code() of the root of v, from v itself, so that it does not hang on the root's rounding: r <= 1.75 2^k exactly where
// v <= 3.0625 4^k (a square that FP32 holds, and the next larger v has a root that rounds to more than 1.75 2^k).  3.0625 4^k
// has the bits ((2 k + 128) << 23) + 0x440000, so the least such k is ((bits - 0x440001) >> 24) - 63, and the code 119 + k.
__device__ __forceinline__ uint32_t root_scale_code(uint32_t v_bits) { return v_bits < 0x00800000u ? 127u : ((v_bits - 0x440001u) >> 24) + 56u; }

// Root y = r / scale, 0 <= y <= 448, on the E4M3 grid, at least its least step 2^-9 unless y = 0.
// Stochastic: 16 random bits are added below the three fraction bits and the rest is cut off; below 2^-6, where the
// grid is even, the same is done at y + 2^-6, whose unit is that grid's.
template <bool kStochastic>
__device__ __forceinline__ float root_on_grid(float y, uint32_t noise) {
  float q = y;
  if constexpr (kStochastic) {
    const float base = y < 0.015625f ? 0.015625f : 0.f;
    q = __uint_as_float((__float_as_uint(y + base) + ((noise & 0xFFFF0000u) >> 12)) & 0xFFF00000u) - base;
  }
  return y > 0.f ? fmaxf(q, 0.001953125f) : y;
}
// BF16 by adding 16 random bits below it and cutting off the rest; infinities stay as they are, NaN is kept from the carry.
__device__ __forceinline__ float bf16_stochastic(float p, uint32_t noise) {
  const float q = __uint_as_float((__float_as_uint(p) + (noise & 0xFFFFu)) & 0xFFFF0000u);
  return p == p ? q : p;
}

// One lane's four elements of a block, by pointers to them: the blocks of a piece lie at fixed distances.
template <class P, class G, bool kEight>
struct Lane {
  using State = typename std::conditional<kEight, uint8_t, float>::type;
  P* p;
  const G* g;
  State *m, *v;
  __nv_bfloat16* copy;   // may be NULL
  uint8_t *m_scale, *v_scale;
  uint32_t index;        // of the first element, modulo 2^32: part of the hash
  __device__ __forceinline__ Lane(const Entry& e, int64_t at, int lane) {
    const int64_t i = at + lane * 4;
    p = static_cast<P*>(e.param) + i, g = static_cast<const G*>(e.grad) + i, m = static_cast<State*>(e.m) + i, v = static_cast<State*>(e.v) + i;
    copy = sizeof(P) == 4 && e.copy ? e.copy + i : nullptr;
    if constexpr (kEight) m_scale = e.m_scale + at / kBlock, v_scale = e.v_scale + at / kBlock;
    index = (uint32_t)i;
  }
};
template <class P, class G, bool kEight>
struct Block {
  using L = Lane<P, G, kEight>;
  Raw<P> p;
  Raw<G> g;
  Raw<typename L::State> m, v;
  uint32_t m_scale, v_scale;
  __device__ __forceinline__ void load(const L& l, int b, bool vec, int64_t left) {
    p.load(l.p + b * kBlock, vec, left);
    g.load(l.g + b * kBlock, vec, left);
    m.load(l.m + b * kBlock, vec, left);
    v.load(l.v + b * kBlock, vec, left);
    if constexpr (kEight) m_scale = l.m_scale[b], v_scale = l.v_scale[b];
  }
};

// One block; returns the codes of its new scales (m in the low half, v in the high half).
template <class P, class G, bool kEight, bool kStochastic>
__device__ __forceinline__ uint32_t update(const Step& t, const Lane<P, G, kEight>& l, const Block<P, G, kEight>& x, int b, bool vec, int64_t left, float clip, uint32_t key) {
  const Pair clip2 = pair(clip, clip), b1 = pair(t.beta1, t.beta1), c1 = pair(t.one_minus_beta1, t.one_minus_beta1), b2 = pair(t.beta2, t.beta2),
             c2 = pair(t.one_minus_beta2, t.one_minus_beta2);
  float p[4], m[4], v[4], r[4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const Pair g = (h ? x.g.hi() : x.g.lo()) * clip2;
    Pair m2 = h ? x.m.hi() : x.m.lo(), v2 = h ? x.v.hi() : x.v.lo();
    if constexpr (kEight) {
      const float sm = scale_value(x.m_scale), sv = scale_value(x.v_scale);
      m2 = m2 * pair(sm, sm), v2 = v2 * pair(sv, sv);
      v2 = v2 * v2;   // the state is the root
    }
    // every product and sum is rounded by itself: the rounding to 8 bits after it then does not hang on a contraction
    m2 = m2 * b1 + g * c1;
    v2 = v2 * b2 + (g * c2) * g;
    const float2 mf = both(m2), vf = both(v2);
    m[2 * h] = mf.x, m[2 * h + 1] = mf.y, v[2 * h] = vf.x, v[2 * h + 1] = vf.y;
    r[2 * h] = root<kEight>(vf.x), r[2 * h + 1] = root<kEight>(vf.y);
    // the step is a few units in the last place off, which is little beside the parameter
    const float2 d = both(multiply_add(pair(r[2 * h], r[2 * h + 1]), pair(t.root_bias, t.root_bias), pair(t.eps, t.eps)));
    const Pair step = m2 * pair(-t.step_size, -t.step_size) * pair(reciprocal(d.x), reciprocal(d.y));
    const float2 pf = both(multiply_add(h ? x.p.hi() : x.p.lo(), pair(t.decay, t.decay), step));
    p[2 * h] = pf.x, p[2 * h + 1] = pf.y;
  }
  uint32_t noise[4] = {};
  if constexpr (kStochastic) {
    mix4((l.index + (uint32_t)(b * kBlock)) ^ key, noise);   // index is a multiple of four
  }
  if constexpr (kStochastic && sizeof(P) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = bf16_stochastic(p[i], noise[i]);
  }
  store4(l.p + b * kBlock, vec, left, p);
  if (sizeof(P) == 4 && l.copy) store4(l.copy + b * kBlock, vec, left, p);
  if constexpr (kEight) {
    // The maxima pass over NaN (m) or show what is not finite as larger than all else (v, whose bits are compared).  An m that is not
    // finite without its v being so can only be a NaN that was there before.
    uint32_t top_m = __float_as_uint(fmaxf(fmaxf(fabsf(m[0]), fabsf(m[1])), fmaxf(fabsf(m[2]), fabsf(m[3])))) & 0x7FFFFFFFu;
    uint32_t top_v = max(max(__float_as_uint(v[0]) & 0x7FFFFFFFu, __float_as_uint(v[1]) & 0x7FFFFFFFu), max(__float_as_uint(v[2]) & 0x7FFFFFFFu, __float_as_uint(v[3]) & 0x7FFFFFFFu));
    top_m = __reduce_max_sync(0xFFFFFFFFu, top_m), top_v = __reduce_max_sync(0xFFFFFFFFu, top_v);
    if (max(top_m, top_v) >= 0x7F800000u) {
      // something is not finite (the same for the whole warp): it becomes NaN and stays out of the scales
      top_m = max(max(finite_bits(m[0]), finite_bits(m[1])), max(finite_bits(m[2]), finite_bits(m[3])));
      top_v = max(max(finite_bits(v[0]), finite_bits(v[1])), max(finite_bits(v[2]), finite_bits(v[3])));
      top_m = __reduce_max_sync(0xFFFFFFFFu, top_m), top_v = __reduce_max_sync(0xFFFFFFFFu, top_v);
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] -= m[i] - m[i], r[i] -= r[i] - r[i];   // subtracted: a negative zero keeps its sign
    }
    const uint32_t code_m = scale_code(top_m), code_r = root_scale_code(top_v);
    const float im = scale_recip(code_m), ir = scale_recip(code_r);
    store4(l.m + b * kBlock, vec, left, pack4(m[0] * im, m[1] * im, m[2] * im, m[3] * im));
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = root_on_grid<kStochastic>(r[i] * ir, noise[i]);
    store4(l.v + b * kBlock, vec, left, pack4(r[0], r[1], r[2], r[3]));
    return code_m | code_r << 16;
  } else {
    store4(l.m + b * kBlock, vec, left, m);
    store4(l.v + b * kBlock, vec, left, v);
    return 0;
  }
}

template <class P, class G, bool kEight, bool kStochastic, int kTensors>
__global__ void __launch_bounds__(256, !kEight ? 2 : sizeof(P) == 4 ? 3 : 4) adamw_kernel(const __grid_constant__ Table<kTensors> t) {
  if (t.skip && *t.skip) return;
  const float clip = t.grad_scale ? *t.grad_scale : 1.f;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  // the warps of the whole grid sweep the pieces together: what is read and written at one time lies close together
  int at_tensor = 0;
  for (uint32_t piece = blockIdx.x * 8 + warp; piece < t.pieces; piece += gridDim.x * 8) {
    int hi = t.count;   // the tensor whose pieces hold this one: not before the last one's
    while (hi - at_tensor > 1) {
      const int mid = (at_tensor + hi) / 2;
      if (t.first_piece[mid] <= piece) at_tensor = mid; else hi = mid;
    }
    const Entry& e = t.entry[at_tensor];
    const bool aligned = e.n > 0;
    const int64_t n = aligned ? e.n : -e.n, at = (int64_t)(piece - t.first_piece[at_tensor]) * kPiece;
    const uint32_t key = mix(t.first_tensor + (uint32_t)at_tensor + 1u) ^ t.seed_key;
    if (aligned && at + kPiece <= n) {
      const Lane<P, G, kEight> l(e, at, lane);
      Block<P, G, kEight> x[kPieceBlocks];
      uint32_t codes = 0;
#pragma unroll
      for (int b = 0; b < kPieceBlocks; ++b) x[b].load(l, b, true, 4);
#pragma unroll
      for (int b = 0; b < kPieceBlocks; ++b) {
        const uint32_t c = update<P, G, kEight, kStochastic>(t, l, x[b], b, true, 4, clip, key);
        if (lane == b) codes = c;
      }
      // the scales of the four blocks in one request each: single bytes, one request at a time, cost 0.28 of 0.97 ms over 256 M parameters
      if (kEight && lane < kPieceBlocks) l.m_scale[lane] = (uint8_t)codes, l.v_scale[lane] = (uint8_t)(codes >> 16);
    } else {
#pragma unroll 1
      for (int64_t a = at; a < n && a < at + kPiece; a += kBlock) {
        const bool vec = aligned && a + kBlock <= n;
        const int64_t left = n - a - lane * 4;
        const Lane<P, G, kEight> l(e, a, lane);
        Block<P, G, kEight> x;
        x.load(l, 0, vec, left);
        const uint32_t c = update<P, G, kEight, kStochastic>(t, l, x, 0, vec, left, clip, key);
        if (kEight && lane == 0) *l.m_scale = (uint8_t)c, *l.v_scale = (uint8_t)(c >> 16);
      }
    }
  }
}

template <class P, class G, int kTensors>
cudaError_t launch(const Table<kTensors>& t, bool eight, bool stochastic, unsigned blocks, cudaStream_t st) {
  if (eight)
    stochastic ? adamw_kernel<P, G, true, true><<<blocks, 256, 0, st>>>(t) : adamw_kernel<P, G, true, false><<<blocks, 256, 0, st>>>(t);
  else
    stochastic ? adamw_kernel<P, G, false, true><<<blocks, 256, 0, st>>>(t) : adamw_kernel<P, G, false, false><<<blocks, 256, 0, st>>>(t);
  return cudaGetLastError();
}

bool aligned_to(const void* p, int a) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(a - 1)) == 0; }

// One launch over `count` <= kTensors of the caller's tensors, from `first` on.
template <int kTensors>
cudaError_t run(const Step& step, const ozk_adamw_tensor* tensors, int64_t first, int count, const ozk_adamw_options* o, cudaStream_t st) {
  const int ps = o->param_type == OZK_F32 ? 4 : 2, gs = o->grad_type == OZK_F32 ? 4 : 2, ss = o->state_bits == 8 ? 1 : 4;
  Table<kTensors> t;
  static_cast<Step&>(t) = step;
  t.count = count;
  t.first_tensor = (uint32_t)first;
  uint32_t pieces = 0;
  for (int i = 0; i < count; ++i) {
    const ozk_adamw_tensor& x = tensors[first + i];
    const bool vec = aligned_to(x.param, 4 * ps) && aligned_to(x.grad, 4 * gs) && aligned_to(x.m, 4 * ss) && aligned_to(x.v, 4 * ss) && aligned_to(x.copy, 8);
    t.entry[i] = Entry{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, static_cast<__nv_bfloat16*>(x.copy), vec ? x.n : -x.n};
    t.first_piece[i] = pieces;
    pieces += (uint32_t)ceil_div(x.n, kPiece);
  }
  t.first_piece[count] = pieces;
  t.pieces = pieces;
  if (pieces == 0) return cudaSuccess;
  // a warp for every piece; from 32 thread blocks per multiprocessor on (eight to sixteen times what runs at a time) each takes several
  const int64_t most = (int64_t)device_sm_count() * 32, wanted = ceil_div(pieces, 8);
  const unsigned blocks = (unsigned)(wanted < most ? wanted : most);
  const bool eight = o->state_bits == 8, stochastic = o->stochastic && (eight || o->param_type == OZK_BF16);
  if (o->param_type == OZK_F32)
    return o->grad_type == OZK_F32 ? launch<float, float>(t, eight, stochastic, blocks, st) : launch<float, __nv_bfloat16>(t, eight, stochastic, blocks, st);
  return o->grad_type == OZK_F32 ? launch<__nv_bfloat16, float>(t, eight, stochastic, blocks, st) : launch<__nv_bfloat16, __nv_bfloat16>(t, eight, stochastic, blocks, st);
}

}  // namespace
}  // namespace ozk

using namespace ozk;

extern "C" ozk_status ozk_adamw_step(const ozk_adamw_tensor* tensors, int64_t count, const ozk_adamw_options* o, void* stream) {
  if (count < 0 || !o || (count > 0 && !tensors)) return OZK_ERR_INVALID_ARG;
  if ((o->param_type != OZK_F32 && o->param_type != OZK_BF16) || (o->grad_type != OZK_F32 && o->grad_type != OZK_BF16) ||
      (o->state_bits != 8 && o->state_bits != 32) || (o->stochastic != 0 && o->stochastic != 1) || o->step < 1)
    return OZK_ERR_INVALID_ARG;
  if (!(o->beta1 >= 0 && o->beta1 < 1) || !(o->beta2 >= 0 && o->beta2 < 1) || !(o->eps >= 0) || !(o->lr >= 0) || !(o->weight_decay >= 0))
    return OZK_ERR_INVALID_ARG;
  if (!aligned_to(o->grad_scale, 4) || !aligned_to(o->skip, 4)) return OZK_ERR_INVALID_ARG;
  const int ps = o->param_type == OZK_F32 ? 4 : 2, gs = o->grad_type == OZK_F32 ? 4 : 2, ss = o->state_bits == 8 ? 1 : 4;
  for (int64_t i = 0; i < count; ++i) {
    const ozk_adamw_tensor& x = tensors[i];
    if (x.n < 0) return OZK_ERR_INVALID_ARG;
    if (x.n == 0) continue;
    if (!x.param || !x.grad || !x.m || !x.v || !aligned_to(x.param, ps) || !aligned_to(x.grad, gs) || !aligned_to(x.m, ss) || !aligned_to(x.v, ss))
      return OZK_ERR_INVALID_ARG;
    if (o->state_bits == 8 && (!x.m_scale || !x.v_scale)) return OZK_ERR_INVALID_ARG;
    if (x.copy && (o->param_type != OZK_F32 || !aligned_to(x.copy, 2))) return OZK_ERR_INVALID_ARG;
    if (ceil_div(x.n, kPiece) > INT32_MAX) return OZK_ERR_UNSUPPORTED;   // the pieces of a launch are counted in 31 bits
  }
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Step t;
  t.grad_scale = o->grad_scale;
  t.skip = o->skip;
  t.beta1 = (float)o->beta1, t.one_minus_beta1 = (float)(1.0 - o->beta1);
  t.beta2 = (float)o->beta2, t.one_minus_beta2 = (float)(1.0 - o->beta2);
  t.decay = (float)(1.0 - o->lr * o->weight_decay);
  t.step_size = (float)(o->lr / (1.0 - pow(o->beta1, (double)o->step)));
  t.root_bias = (float)(1.0 / sqrt(1.0 - pow(o->beta2, (double)o->step)));
  t.eps = (float)o->eps;
  t.seed_key = mix(o->seed);
  for (int64_t first = 0; first < count;) {
    int here = 0;
    for (int64_t pieces = 0; here < kMostTensors && first + here < count; ++here) {
      pieces += ceil_div(tensors[first + here].n, kPiece);
      if (pieces > INT32_MAX) break;
    }
    const cudaError_t e = here <= kFewTensors ? run<kFewTensors>(t, tensors, first, here, o, st) : run<kMostTensors>(t, tensors, first, here, o, st);
    if (e != cudaSuccess) return OZK_ERR_CUDA;
    first += here;
  }
  return OZK_OK;
}
