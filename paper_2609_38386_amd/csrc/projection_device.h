// Device functions of the projection kernels: outputs, activations, 4-bit weights.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2_t v;
  v[0] = (__bf16)lo;
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}

// act(g) u, the activation in fp32, then the product.  e^-y is 2^(y log2 e) with the product's
// rounding error put back, so that SiLU's gates far below 0, whose weight is all in the power, are
// 4 fp32 steps (2^-23) off at most; GELU's y is itself a rounded one, whose error counts |y| times
// there (7 |y| half steps).  Where the power is past 2^125, 1 / (1 + e^-y) is e^y to the last bit
// and its reciprocal would leave fp32's normal range before the activation does (g = -88: -5e-37):
// 2^64 e^y is multiplied by the gate first.
__device__ __forceinline__ float gated(float g, float u, int act) {
  const float y = act ? 1.5957691216057308f * (g + 0.044715f * g * g * g) : g;
  constexpr float LOG2E = 1.44269504088896f, LOG2E_LOW = 1.925963033500e-8f;
  const float t = -y * LOG2E;
  const float rest = __builtin_fmaf(-y, LOG2E, -t) - y * LOG2E_LOW;
  const bool far = t > 125.f;
  float shifted;
  {
#pragma clang fp contract(off)
    shifted = 64.f - t;  // (exact there, of t as it was rounded: `rest` belongs to that one)
  }
  float e = __builtin_amdgcn_exp2f(far ? shifted : t);
  // (the power of an infinite y stays as it is)
  const float turn = rest * 0.693147181f;
  e = __builtin_fabsf(rest) < 1.f ? __builtin_fmaf(e, far ? -turn : turn, e) : e;
  return (far ? g * e * 0x1p-64f : g * __builtin_amdgcn_rcpf(1.f + e)) * u;
}

// The eight weights of a dword of codes in the scale of an exponent byte, exact for
// every bf16 value; byte 255 gives NaN.
__device__ __forceinline__ bf16x8_t widen(uint32_t codes, float scale) {
  union {
    bf16x2_t p[4];
    bf16x8_t v;
  } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return r.v;
}
// The conversion reads the scale's exponent field alone.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}

}  // namespace
