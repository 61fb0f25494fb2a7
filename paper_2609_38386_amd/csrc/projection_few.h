// Projections of few tokens: weights and tokens through LDS, by copies of whole row segments,
// into v_mfma_f32_16x16x32_bf16 as out^T = W x^T.
//
// A workgroup takes BLOCKS blocks of 16 rows of weights (gated: rows of the gate and of the up
// in turn) and TOKENS tokens.  Its wavefronts (and, with splits, several workgroups) share K,
// each through a ring of its own without barriers, and their results are added through LDS, in
// wavefront order.
//
// Why through LDS: as operands come, neighbouring lanes hold 16 bytes of different rows, and a
// load of 64 such pieces keeps the address unit busy four times as long as a copy of whole row
// segments (weights and tokens straight from memory into registers: 1 token of 4096 x 12288
// in 4 bits 10.7 us with any number of loads in flight, this way 7.4).  Products of 16 x 16
// leave the fewest idle columns to 1-16 tokens and need half the operand reads of 32 x 32.
//
// Bound by memory: a compute unit's copies in flight are limited, and those of weights and of tokens
// share them.  Few tokens run near the card's rate (2 x 12288 x 4096 bf16, 8 tokens: 32-34 us,
// 6.0-6.3 TB/s), 16-32 tokens of few features below it: 32 of 5120 x 25600 in 4 bits take 23.6 us for
// 72 MB of weights from HBM (17.9 where the caches have them) and, over all tiles, 131 MB of tokens
// from L2, where the weights' copies alone take 17.0, the tokens' 11.9, both without most products
// 22.7.  (The call is 25.8 us with the sum of its three parts, 20.1 from the caches.)
#pragma once

#include "projection_tiles.h"

namespace {

// A workgroup's unit: its tile's first feature and token, and its part of the steps of K, which
// its wavefronts take in turn (so that they read neighbouring pieces of a row at about the same
// time: 32 tokens of 5120 x 25600 in 4 bits, weights from HBM, took 0.95 of the launch with
// neighbouring steps for each).  Divisions only where there is something to divide (0.1-0.2 us of a
// launch of 3).
struct Unit {
  uint32_t tile, part;
  int n0, m0, from, to;
};
template <int FEATURES, int TOKENS>
__device__ __forceinline__ Unit unit_of(const dlfp::ProjectionArgs& a, dlfp::Split split,
                                        int steps) {
  Unit r{blockIdx.x, 0, 0, 0, 0, steps};
  if (split.splits > 1) {
    r.tile = blockIdx.x / split.splits;
    r.part = blockIdx.x - r.tile * split.splits;
    r.from = (uint32_t)steps * r.part / split.splits;
    r.to = (uint32_t)steps * (r.part + 1) / split.splits;
  }
  uint32_t across = r.tile;
  if (a.m > TOKENS) {
    const uint32_t gn = (uint32_t)(a.n + FEATURES - 1) / FEATURES, down = r.tile / gn;
    across -= down * gn;
    r.m0 = (int)down * TOKENS;
  }
  r.n0 = (int)across * FEATURES;
  return r;
}

// Four features of a token.
__device__ __forceinline__ void store4(const dlfp::ProjectionArgs& a, int m, int n, f32x4_t v) {
  const int64_t at = (int64_t)m * a.ldo + n;
  if (a.out_f32)
    *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + at) = v;
  else
    *reinterpret_cast<u32x2_t*>(static_cast<uint16_t*>(a.out) + at) =
        u32x2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// The end of a unit, when its wavefront is done: lane l holds features 4 (l / 16) .. + 3 of
// token l % 16 of a block.
template <int BLOCKS, int TOKENS, int WAVES, bool GATED, int TB>
__device__ __forceinline__ void store_few(const dlfp::ProjectionArgs& a, dlfp::Split split,
                                          f32x4_t (&acc)[BLOCKS][TB], char* smem, int tid,
                                          int wave, const Unit& own) {
  const int lane = tid & 63;
  wait_copies_barrier<0>();
  f32x4_t* sums = reinterpret_cast<f32x4_t*>(smem);
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int u = 0; u < TB; ++u) sums[((wave * BLOCKS + b) * TB + u) * 64 + lane] = acc[b][u];
  __syncthreads();
  constexpr int OUT = GATED ? BLOCKS / 2 : BLOCKS;
  for (int i = tid; i < OUT * TB * 64; i += 64 * WAVES) {
    const int l = i & 63, u = (i >> 6) % TB, r = (i >> 6) / TB;
    auto sum = [&](int b) {
      f32x4_t v = sums[(b * TB + u) * 64 + l];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) v += sums[((w * BLOCKS + b) * TB + u) * 64 + l];
      return v;
    };
    f32x4_t v = sum(GATED ? 2 * r : r);
    if (split.splits > 1) {
      // Unit (r, u, l) of the gate, then of the up.
      const int64_t at = (int64_t)own.part * (gridDim.x / split.splits) + own.tile;
      f32x4_t* out = reinterpret_cast<f32x4_t*>(split.part) + at * (BLOCKS * TB * 64) + i;
      *out = v;
      if constexpr (GATED) out[OUT * TB * 64] = sum(2 * r + 1);
      continue;
    }
    if constexpr (GATED) v = gated4(v, sum(2 * r + 1), a.act);
    const int tok = 16 * u + (l & 15), m = own.m0 + tok, n = own.n0 + 16 * r + 4 * (l >> 4);
    if (tok < TOKENS && m < a.m && n < a.n) store4(a, m, n, v);
  }
}

// p[0] + p[step] + ... in that order, of SPLITS addresses: all of them are read before the first
// is waited for (47 tokens of 128 x 14016 in 8 parts: one after the other 7.5 us, this way 6.3).
template <int SPLITS, int UNITS>
__device__ __forceinline__ void sum_parts(f32x4_t (&v)[UNITS], const f32x4_t* p, int64_t step,
                                          int unit_step) {
  f32x4_t parts[SPLITS][UNITS];
#pragma unroll
  for (int s = 0; s < SPLITS; ++s)
#pragma unroll
    for (int i = 0; i < UNITS; ++i) parts[s][i] = p[s * step + i * unit_step];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    v[i] = parts[0][i];
#pragma unroll
    for (int s = 1; s < SPLITS; ++s) v[i] += parts[s][i];
  }
}
template <int UNITS>
__device__ __forceinline__ void sum_splits(f32x4_t (&v)[UNITS], const f32x4_t* p, int64_t step,
                                           int unit_step, int splits) {
  switch (splits) {
    case 2: return sum_parts<2>(v, p, step, unit_step);
    case 3: return sum_parts<3>(v, p, step, unit_step);
    case 4: return sum_parts<4>(v, p, step, unit_step);
    case 6: return sum_parts<6>(v, p, step, unit_step);
    default: return sum_parts<8>(v, p, step, unit_step);
  }
}

// The sum of the splits of a tile, in split order: a thread for each unit of the output.
template <int BLOCKS, int TOKENS, bool GATED>
__global__ __launch_bounds__(64) void sum_few_kernel(dlfp::ProjectionArgs a, int gn, int tiles,
                                                     dlfp::Split split) {
  constexpr int TB = TOKENS < 16 ? 1 : TOKENS / 16, OUT = GATED ? BLOCKS / 2 : BLOCKS;
  const int i = blockIdx.x % (OUT * TB), t = blockIdx.x / (OUT * TB), l = threadIdx.x;
  const int u = i % TB, r = i / TB, tok = 16 * u + (l & 15);
  const int m = t / gn * TOKENS + tok, n = t % gn * (16 * OUT) + 16 * r + 4 * (l >> 4);
  if (tok >= TOKENS || m >= a.m || n >= a.n) return;
  constexpr int UNITS = BLOCKS * TB * 64;
  const f32x4_t* p = reinterpret_cast<const f32x4_t*>(split.part) + (int64_t)t * UNITS + i * 64 + l;
  f32x4_t v[GATED ? 2 : 1];
  sum_splits(v, p, (int64_t)tiles * UNITS, OUT * TB * 64, split.splits);
  if constexpr (GATED) v[0] = gated4(v[0], v[1], a.act);
  store4(a, m, n, v[0]);
}

}  // namespace
