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

// The power of an activation, e^-y, is 2^(t + rest): t the product -y log2 e as it is rounded, rest
// its rounding error, so that SiLU's gates far below 0, whose weight is all in the power, are 4 fp32
// steps (2^-23) off at most.  (GELU's y is itself a rounded one, whose error counts |y| times
// there: 7 |y| half steps.)
struct Power {
  float t, rest;
};
__device__ __forceinline__ Power power_of(float g, int act) {
  const float y = act ? 1.5957691216057308f * (g + 0.044715f * g * g * g) : g;
  constexpr float LOG2E = 1.44269504088896f, LOG2E_LOW = 1.925963033500e-8f;
  const float t = -y * LOG2E;
  return {t, __builtin_fmaf(-y, LOG2E, -t) - y * LOG2E_LOW};
}
// 2^(t + rest); of an infinite t, whose rest is NaN, 2^t.
__device__ __forceinline__ float raise(float t, float rest) {
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_fabsf(rest) < 1.f ? __builtin_fmaf(e, rest * 0.693147181f, e) : e;
}

// act(g) u of four features, the activation in fp32, then the product.
//
// Where the power is past 2^125, 1 / (1 + e^-y) is e^y to the last bit, and the reciprocal would
// leave fp32's normal range before the activation does (SiLU of -88.5 is -3.2e-37): 2^64 e^y is
// multiplied by the gate first.  One branch for four, since hardly a gate is there (as selections
// for each it took 3-5% of a launch of short K, 2048 tokens of 2 x 2816 x 1024 29.6 -> 31.0 us).
__device__ __forceinline__ f32x4_t gated4(f32x4_t g, f32x4_t u, int act) {
  f32x4_t v;
  Power p[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    p[j] = power_of(g[j], act);
    v[j] = g[j] * __builtin_amdgcn_rcpf(1.f + raise(p[j].t, p[j].rest)) * u[j];
  }
  const float most =
      __builtin_fmaxf(__builtin_fmaxf(p[0].t, p[1].t), __builtin_fmaxf(p[2].t, p[3].t));
  if (__builtin_expect(most > 125.f, 0)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma clang fp contract(off)
      const float t = 64.f - p[j].t;  // (exact there, of t as it was rounded: `rest` is that one's)
      if (p[j].t > 125.f) v[j] = g[j] * raise(t, -p[j].rest) * 0x1p-64f * u[j];
    }
  }
  return v;
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
