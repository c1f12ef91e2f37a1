// Shared by the 8-bit operators: E4M3 and UE8M0 conversions, element loads, argument checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ozk_common.cuh"

namespace ozk {
namespace fp8 {

constexpr int kBlock = 128;   // elements that share a scale, along the axis a product sums over

// Two floats (|x| <= 448 or NaN) to E4M3, to nearest even; `lo` lands in the low byte.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) { return pack2(a, b) | (pack2(c, d) << 16); }
// Two E4M3 bytes to floats, exactly.
__device__ __forceinline__ float2 unpack2(uint32_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
  float2 f;
  asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
  return f;
}

// Magnitude bits of x if it is finite, else 0: amax over a block is an integer maximum of these.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}
// UE8M0 code of the least power of two 2^e >= 2^-127 with amax <= 448 * 2^e (127, i.e. 1, for a block of zeros).
// With amax = f 2^E, 1 <= f < 2, and 448 = 1.75 * 2^8: e = E - 8 + (f > 1.75), the last by a carry out of the fraction bits.
__device__ __forceinline__ uint32_t scale_code(uint32_t amax_bits) {
  return amax_bits == 0 ? 127u : (uint32_t)max((int)((amax_bits + 0x1FFFFFu) >> 23) - 8, 0);
}
// 2^(c - 127) and its reciprocal; c = 0 is the subnormal 2^-127.
__device__ __forceinline__ float scale_value(uint32_t c) { return __uint_as_float(max(c << 23, 1u << 22)); }
__device__ __forceinline__ float scale_recip(uint32_t c) { return __uint_as_float((254u - c) << 23); }   // c <= 247 from scale_code
// x / scale where x is finite, else NaN: x - x is 0 or NaN.  Subtracted, so that a negative zero keeps its sign.
__device__ __forceinline__ float scaled(float x, float recip) { return fmaf(x, recip, -(x - x)); }

// Pairs of floats, multiplied in one instruction; each operation rounds both by itself, as the scalar one does.
struct Pair {
  uint64_t v;
};
__device__ __forceinline__ Pair pair(float lo, float hi) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ float2 both(Pair p) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p.v));
  return f;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float load_element(const float* p) { return *p; }
__device__ __forceinline__ float load_element(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_element(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_element(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace fp8
}  // namespace ozk
