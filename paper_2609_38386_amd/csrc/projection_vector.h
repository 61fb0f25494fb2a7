// Projections of few tokens: weights straight from memory into the operands of
// v_mfma_f32_16x16x32_bf16, computed as out^T = W x^T.
//
// A workgroup takes 16 ROWS features and 16 tokens; its wavefronts take 128-deep K
// steps in turn and their results are added through LDS, in wavefront order.  Of a
// step, lane l takes row l % 16 of each 16-row block and, with 4-bit weights, the 32
// columns from 32 (l / 16): 16 bytes of codes, a whole group, which are the operands
// of four products.  Which columns a product takes is free as long as both operands
// agree, so that the codes need no other layout than their rows.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dlfp_ffn.h"
#include "projection.h"
#include "projection_device.h"

namespace {

constexpr int VSTEP = 128;  // columns of a step

template <bool CODES>
struct StepWeights;
template <>
struct StepWeights<true> {
  u32x4_t codes;
  uint32_t byte;
  __device__ __forceinline__ void load(const char* row, const uint8_t* exps, int k0, int quad,
                                       bool inside) {
    const int c = inside ? k0 + 32 * quad : 0;
    codes = *reinterpret_cast<const u32x4_t*>(row + (c >> 1));
    byte = exps[c >> 5];
    if (!inside) codes = u32x4_t{};
    if (!inside) byte = 0;
  }
  __device__ __forceinline__ bf16x8_t operand(int t) const { return widen(codes[t], scale_of(byte)); }
  static __device__ __forceinline__ int column(int t, int quad) { return 32 * quad + 8 * t; }
};
template <>
struct StepWeights<false> {
  bf16x8_t w[4];
  __device__ __forceinline__ void load(const char* row, const uint8_t*, int k0, int quad,
                                       bool inside) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int c = inside || t < 2 ? k0 + column(t, quad) : 0;
      w[t] = *reinterpret_cast<const bf16x8_t*>(row + 2 * (int64_t)c);
      if (!inside && t >= 2) w[t] = bf16x8_t{};
    }
  }
  __device__ __forceinline__ bf16x8_t operand(int t) const { return w[t]; }
  static __device__ __forceinline__ int column(int t, int quad) { return 32 * t + 8 * quad; }
};

template <bool CODES, bool GATED, int ROWS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void vector_kernel(dlfp::ProjectionArgs a) {
  constexpr int B = ROWS * (GATED ? 2 : 1);  // 16-row weight blocks
  __shared__ __attribute__((aligned(16))) f32x4_t sums[WAVES][B][64];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int lr = lane & 15, quad = lane >> 4;
  const uint32_t gn = (uint32_t)(a.n + 16 * ROWS - 1) / (16 * ROWS);
  const int n0 = (int)(blockIdx.x % gn) * (16 * ROWS), m0 = (int)(blockIdx.x / gn) * 16;
  const char* rows[B];
  const uint8_t* exps[B];
#pragma unroll
  for (int b = 0; b < B; ++b) {
    const int which = GATED ? b & 1 : 0, r = min(n0 + 16 * (GATED ? b >> 1 : b), a.n - 16) + lr;
    rows[b] = static_cast<const char*>(a.weights[which]) +
              (CODES ? (int64_t)r * (a.k >> 1) : (int64_t)r * a.k * 2);
    exps[b] = CODES ? a.exps[which] + (int64_t)r * (a.k >> 5) : nullptr;
  }
  const uint16_t* x = a.x + (int64_t)min(m0 + lr, a.m - 1) * a.ldx;

  f32x4_t acc[B];
#pragma unroll
  for (int b = 0; b < B; ++b) acc[b] = f32x4_t{};
  for (int k0 = VSTEP * wave; k0 < a.k; k0 += VSTEP * WAVES) {
    // Of a last step of 64 columns half of the lanes' columns, with bf16 weights half
    // of the products, are past the row: zeros.
    const bool whole = k0 + VSTEP <= a.k;
    const bool inside = whole || (CODES && quad < 2);
    StepWeights<CODES> w[B];
    bf16x8_t xf[4];
#pragma unroll
    for (int b = 0; b < B; ++b) w[b].load(rows[b], exps[b], k0, quad, inside);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bool in = inside || (!CODES && t < 2);
      xf[t] = *reinterpret_cast<const bf16x8_t*>(
          x + (in ? k0 + StepWeights<CODES>::column(t, quad) : 0));
      if (!in) xf[t] = bf16x8_t{};
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < B; ++b)
        acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[b].operand(t), xf[t], acc[b], 0, 0, 0);
  }

  // Lane l holds features 4 (l / 16) .. + 3 of token l % 16.
#pragma unroll
  for (int b = 0; b < B; ++b) sums[wave][b][lane] = acc[b];
  __syncthreads();
  for (int u = tid; u < ROWS * 64; u += 64 * WAVES) {
    const int r = u >> 6, l = u & 63;
    f32x4_t v = sums[0][GATED ? 2 * r : r][l], up{};
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += sums[w][GATED ? 2 * r : r][l];
    if constexpr (GATED) {
      up = sums[0][2 * r + 1][l];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) up += sums[w][2 * r + 1][l];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = gated(v[j], up[j], a.act);
    }
    const int m = m0 + (l & 15), n = n0 + 16 * r + 4 * (l >> 4);
    if (m >= a.m || n >= a.n) continue;
    const int64_t e = (int64_t)m * a.ldo + n;
    if (a.out_f32)
      *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + e) = v;
    else
      *reinterpret_cast<u32x2_t*>(static_cast<uint16_t*>(a.out) + e) =
          u32x2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  }
}

template <bool CODES, bool GATED, int ROWS, int WAVES>
int launch_vector(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  const int64_t blocks = ((int64_t)a.n + 16 * ROWS - 1) / (16 * ROWS) * (((int64_t)a.m + 15) / 16);
  if (blocks * 64 * WAVES >= (int64_t)1 << 32) return DLFP_ERANGE;
  (void)hipGetLastError();
  vector_kernel<CODES, GATED, ROWS, WAVES><<<(uint32_t)blocks, 64 * WAVES, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

}  // namespace
