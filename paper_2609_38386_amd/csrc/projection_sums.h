// Tiles whose K is split over workgroups: their partial sums and the launch that adds them.
#pragma once

#include "projection_few.h"

namespace {

// A wave's accumulators as units of four features of a token: unit (wave, q, u, g, lane) has
// features 8 g + 4 (lane / 32) .. + 3 of its block q, token lane % 32 of its block u.
template <int BN, int BM>
__device__ __forceinline__ void store_parts(dlfp::Split split, f32x16_t (&acc)[BN][BM],
                                            int64_t wave, int lane) {
  f32x4_t* out = reinterpret_cast<f32x4_t*>(split.part) + wave * (BN * BM * 256) + lane;
#pragma unroll
  for (int q = 0; q < BN; ++q)
#pragma unroll
    for (int u = 0; u < BM; ++u)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        out[((q * BM + u) * 4 + g) * 64] = f32x4_t{acc[q][u][4 * g], acc[q][u][4 * g + 1],
                                                   acc[q][u][4 * g + 2], acc[q][u][4 * g + 3]};
}

// The sum of the splits of a tile, in split order: a thread for each unit of the output.
template <int TN, int TM, int WN, int WM, bool GATED>
__global__ __launch_bounds__(256) void sum_tiles_kernel(dlfp::ProjectionArgs a, int gm, int gn,
                                                        dlfp::Split split) {
  constexpr int BN = TN / WN / 32, BM = TM / WM / 32, GROUPS = GATED ? 2 : 4;
  constexpr int OUT = TN * TM / 16 * GROUPS, UNITS = TN * TM / 4;
  constexpr int BLOCKS = OUT / 256;
  static_assert(OUT % 256 == 0, "whole workgroups");
  const int t = blockIdx.x / BLOCKS;
  int i = (blockIdx.x - t * BLOCKS) * 256 + threadIdx.x;
  const int lane = i & 63, g = (i >> 6) % GROUPS;
  i = (i >> 6) / GROUPS;
  const int u = i % BM, q = i / BM % BN, wave = i / BM / BN;
  constexpr int BAND = 8;
  const int first = t / (BAND * gn) * BAND, h = min(BAND, gm - first), in = t - first * gn;
  const int b = wave / WM * BN + q;
  const int n = (in / h) * (GATED ? TN / 2 : TN) + (GATED ? 16 : 32) * b + 8 * g + 4 * (lane >> 5);
  const int m = (first + in % h) * TM + 32 * (wave % WM * BM + u) + (lane & 31);
  if (m >= a.m || n >= a.n) return;
  const f32x4_t* p = reinterpret_cast<const f32x4_t*>(split.part) + (int64_t)t * UNITS +
                     (((wave * BN + q) * BM + u) * 4 + g) * 64 + lane;
  const int64_t step = (int64_t)gm * gn * UNITS;
  f32x4_t v[GATED ? 2 : 1];
  sum_splits(v, p, step, 2 * 64, split.splits);
  if constexpr (GATED) v[0] = gated4(v[0], v[1], a.act);
  store4(a, m, n, v[0]);
}

}  // namespace
