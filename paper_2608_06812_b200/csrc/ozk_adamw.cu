// One AdamW step over many tensors in one launch, first and second moments in 32 bits or as E4M3 with a scale per 128.
#include <math.h>
#include <string.h>

#include "ozk_fp8.cuh"

namespace ozk {
namespace {

using namespace fp8;

constexpr int kChunk = 4096;        // elements per thread block: eight warps of four blocks of 128
constexpr int kTableTensors = 448;  // tensors per launch: the table travels in the kernel's parameters (at most 32764 bytes)

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
struct Table {
  int count;
  uint32_t first_tensor;              // index in the caller's array of entry 0: part of the hash
  const float* grad_scale;
  const int* skip;
  float beta1, one_minus_beta1, beta2, one_minus_beta2, decay, step_size, root_bias, eps;
  uint32_t seed_key;                  // mix(seed)
  uint32_t first_chunk[kTableTensors + 1];
  Entry entry[kTableTensors];
};
static_assert(sizeof(Table) <= 32764, "kernel parameters");

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

// Four consecutive elements; zeros beyond `left`.
__device__ __forceinline__ void load4(const float* p, bool vec, int64_t left, float (&x)[4]) {
  if (vec) {
    const float4 w = *reinterpret_cast<const float4*>(p);
    x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < left ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, bool vec, int64_t left, float (&x)[4]) {
  if (vec) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    x[0] = bf16_lo(w.x), x[1] = bf16_hi(w.x), x[2] = bf16_lo(w.y), x[3] = bf16_hi(w.y);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < left ? __bfloat162float(p[i]) : 0.f;
  }
}
__device__ __forceinline__ uint32_t load4(const uint8_t* p, bool vec, int64_t left) {
  if (vec) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) w |= (uint32_t)p[i] << (8 * i);
  return w;
}
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

// Root y = r / scale (0 <= y <= 448, or not finite) on the E4M3 grid, at least its least step 2^-9 unless y = 0.
// Stochastic: 16 random bits are added below the three fraction bits and the rest is cut off; below 2^-6, where the
// grid is even, the same is done at y + 2^-6, whose unit is that grid's.
template <bool kStochastic>
__device__ __forceinline__ float root_on_grid(float y, uint32_t noise16) {
  if constexpr (kStochastic) {
    const bool low = y < 0.015625f;
    const float z = low ? y + 0.015625f : y;
    const float w = __uint_as_float((__float_as_uint(z) + (noise16 << 4)) & 0xFFF00000u);
    const float q = low ? w - 0.015625f : w;
    return y > 0.f ? (y <= 448.f ? fmaxf(q, 0.001953125f) : y - y + __uint_as_float(0x7FC00000u)) : y;
  } else {
    return y > 0.f ? (y <= 448.f ? fmaxf(y, 0.001953125f) : __uint_as_float(0x7FC00000u)) : y;
  }
}
// BF16 by adding 16 random bits below it and cutting off the rest; what is not finite stays.
__device__ __forceinline__ float bf16_stochastic(float p, uint32_t noise16) {
  const uint32_t u = __float_as_uint(p);
  return (u & 0x7F800000u) == 0x7F800000u ? p : __uint_as_float((u + noise16) & 0xFFFF0000u);
}

template <class P, class G, bool kEight, bool kStochastic>
__global__ void __launch_bounds__(256) adamw_kernel(const __grid_constant__ Table t) {
  if (t.skip && *t.skip) return;
  // the tensor whose chunks hold this one
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (t.first_chunk[mid] <= blockIdx.x) lo = mid; else hi = mid;
  }
  const Entry& e = t.entry[lo];
  const bool aligned = e.n > 0;
  const int64_t n = aligned ? e.n : -e.n;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t base = (int64_t)(blockIdx.x - t.first_chunk[lo]) * kChunk + warp * (kChunk / 8);
  const float clip = t.grad_scale ? *t.grad_scale : 1.f;
  const uint32_t key = mix(t.first_tensor + (uint32_t)lo + 1u) ^ t.seed_key;
#pragma unroll
  for (int b = 0; b < kChunk / 8 / kBlock; ++b) {
    const int64_t at = base + b * kBlock;
    if (at >= n) break;
    const int64_t i0 = at + lane * 4, left = n - i0;
    const bool vec = aligned && at + kBlock <= n;
    float p[4], g[4], m[4], v[4], r[4];
    load4(static_cast<const P*>(e.param) + i0, vec, left, p);
    load4(static_cast<const G*>(e.grad) + i0, vec, left, g);
    if constexpr (kEight) {
      const uint32_t cm = load4(static_cast<const uint8_t*>(e.m) + i0, vec, left), cv = load4(static_cast<const uint8_t*>(e.v) + i0, vec, left);
      const float sm = scale_value(e.m_scale[at / kBlock]), sv = scale_value(e.v_scale[at / kBlock]);
      const float2 m01 = unpack2(cm & 0xFFFF), m23 = unpack2(cm >> 16), v01 = unpack2(cv & 0xFFFF), v23 = unpack2(cv >> 16);
      m[0] = m01.x * sm, m[1] = m01.y * sm, m[2] = m23.x * sm, m[3] = m23.y * sm;
      v[0] = v01.x * sv, v[1] = v01.y * sv, v[2] = v23.x * sv, v[3] = v23.y * sv;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __fmul_rn(v[i], v[i]);
    } else {
      load4(static_cast<const float*>(e.m) + i0, vec, left, m);
      load4(static_cast<const float*>(e.v) + i0, vec, left, v);
    }
    uint32_t top_m = 0, top_r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // every product and sum rounded by itself: the rounding to 8 bits after it then does not hang on a contraction
      const float gs = __fmul_rn(g[i], clip);
      m[i] = __fadd_rn(__fmul_rn(m[i], t.beta1), __fmul_rn(gs, t.one_minus_beta1));
      v[i] = __fadd_rn(__fmul_rn(v[i], t.beta2), __fmul_rn(__fmul_rn(gs, t.one_minus_beta2), gs));
      r[i] = __fsqrt_rn(v[i]);
      const float u = __fdiv_rn(m[i], __fadd_rn(__fmul_rn(r[i], t.root_bias), t.eps));
      p[i] = __fsub_rn(__fmul_rn(p[i], t.decay), __fmul_rn(u, t.step_size));
      if constexpr (kEight) top_m = max(top_m, finite_bits(m[i])), top_r = max(top_r, finite_bits(r[i]));
    }
    uint32_t noise[4] = {};
    if constexpr (kStochastic) {
#pragma unroll
      for (int i = 0; i < 4; ++i) noise[i] = mix((uint32_t)(i0 + i) ^ key);
    }
    if constexpr (kStochastic && sizeof(P) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = bf16_stochastic(p[i], noise[i] & 0xFFFFu);
    }
    store4(static_cast<P*>(e.param) + i0, vec, left, p);
    if (e.copy) store4(e.copy + i0, vec, left, p);
    if constexpr (kEight) {
      const uint32_t code_m = scale_code(__reduce_max_sync(0xFFFFFFFFu, top_m)), code_r = scale_code(__reduce_max_sync(0xFFFFFFFFu, top_r));
      const float im = scale_recip(code_m), ir = scale_recip(code_r);
      store4(static_cast<uint8_t*>(e.m) + i0, vec, left, pack4(scaled(m[0], im), scaled(m[1], im), scaled(m[2], im), scaled(m[3], im)));
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = root_on_grid<kStochastic>(__fmul_rn(r[i], ir), noise[i] >> 16);
      store4(static_cast<uint8_t*>(e.v) + i0, vec, left, pack4(r[0], r[1], r[2], r[3]));
      if (lane == 0) e.m_scale[at / kBlock] = (uint8_t)code_m, e.v_scale[at / kBlock] = (uint8_t)code_r;
    } else {
      store4(static_cast<float*>(e.m) + i0, vec, left, m);
      store4(static_cast<float*>(e.v) + i0, vec, left, v);
    }
  }
}

template <class P, class G>
cudaError_t launch(const Table& t, bool eight, bool stochastic, unsigned blocks, cudaStream_t st) {
  if (eight)
    stochastic ? adamw_kernel<P, G, true, true><<<blocks, 256, 0, st>>>(t) : adamw_kernel<P, G, true, false><<<blocks, 256, 0, st>>>(t);
  else
    stochastic ? adamw_kernel<P, G, false, true><<<blocks, 256, 0, st>>>(t) : adamw_kernel<P, G, false, false><<<blocks, 256, 0, st>>>(t);
  return cudaGetLastError();
}

bool aligned_to(const void* p, int a) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(a - 1)) == 0; }

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
    if (ceil_div(x.n, kChunk) > INT32_MAX / kTableTensors) return OZK_ERR_UNSUPPORTED;   // chunks of a launch are counted in 31 bits
  }
  if (!device_is_sm100()) return OZK_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Table t;
  t.grad_scale = o->grad_scale;
  t.skip = o->skip;
  t.beta1 = (float)o->beta1, t.one_minus_beta1 = (float)(1.0 - o->beta1);
  t.beta2 = (float)o->beta2, t.one_minus_beta2 = (float)(1.0 - o->beta2);
  t.decay = (float)(1.0 - o->lr * o->weight_decay);
  t.step_size = (float)(o->lr / (1.0 - pow(o->beta1, (double)o->step)));
  t.root_bias = (float)(1.0 / sqrt(1.0 - pow(o->beta2, (double)o->step)));
  t.eps = (float)o->eps;
  t.seed_key = mix(o->seed);
  for (int64_t first = 0; first < count; first += kTableTensors) {
    t.count = (int)(count - first < kTableTensors ? count - first : kTableTensors);
    t.first_tensor = (uint32_t)first;
    uint32_t chunks = 0;
    for (int i = 0; i < t.count; ++i) {
      const ozk_adamw_tensor& x = tensors[first + i];
      const bool vec = aligned_to(x.param, 4 * ps) && aligned_to(x.grad, 4 * gs) && aligned_to(x.m, 4 * ss) && aligned_to(x.v, 4 * ss) && aligned_to(x.copy, 8);
      t.entry[i] = Entry{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, static_cast<__nv_bfloat16*>(x.copy), vec ? x.n : -x.n};
      t.first_chunk[i] = chunks;
      chunks += (uint32_t)ceil_div(x.n, kChunk);
    }
    t.first_chunk[t.count] = chunks;
    if (chunks == 0) continue;
    const bool eight = o->state_bits == 8, stochastic = o->stochastic && (eight || o->param_type == OZK_BF16);
    cudaError_t e;
    if (o->param_type == OZK_F32)
      e = o->grad_type == OZK_F32 ? launch<float, float>(t, eight, stochastic, chunks, st) : launch<float, __nv_bfloat16>(t, eight, stochastic, chunks, st);
    else
      e = o->grad_type == OZK_F32 ? launch<__nv_bfloat16, float>(t, eight, stochastic, chunks, st)
                                  : launch<__nv_bfloat16, __nv_bfloat16>(t, eight, stochastic, chunks, st);
    if (e != cudaSuccess) return OZK_ERR_CUDA;
  }
  return OZK_OK;
}
