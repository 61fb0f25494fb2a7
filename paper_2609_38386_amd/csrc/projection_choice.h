// Which kernel and tile a projection takes, and over how many workgroups K is split: those
// whose estimated time is lowest.
//
// K over workgroups pays where the tiles leave compute units empty (5120 x 25600 in 4 bits, weights
// from HBM, the forms that are taken without a workspace and with one: 256 tokens 106 us whole, 70
// in 6 parts; 128: 75 and 47; 32: 38.7 and 25.8); it costs the second launch's 2-3 us and the
// partial sums' bytes twice.  A second launch and not the last of a tile's workgroups adds them: it
// needs no counters that someone has to have zeroed.
#pragma once

#include <algorithm>
#include <cstdint>

#include "dlfp.h"
#include "projection.h"

namespace {

// `down` x `across` tiles of tokens and features.
struct Grid {
  int64_t down, across;
};
typedef int (*Launch)(const dlfp::ProjectionArgs&, Grid, dlfp::Split, hipStream_t);

// A tile of `rows` rows of weights and `tokens` tokens, of one workgroup of `threads`.  Its
// wavefronts share steps of `columns` columns, or take all of them (waves 0).  `lds` bytes besides
// the exponents of `blocks` blocks, where that matters (blocks > 0).
//
// Time in microseconds, with u = tiles times splits / 256, s = steps of a unit (of a wavefront
// where they share them, of 64 columns otherwise) and b = MB of weights:
//   c0 + c1 s + (c2 + c3 s) u + (c4 + c5 s) ceil(u) + c6 b + (c7 + c8 s) ceil(u / resident)
// and with splits + c9 + c10 times the MB of partial sums, where `resident` workgroups fit a
// compute unit (0: left out), and where wavefronts share the steps + c11 times the MB of tokens
// that the L2s read (each all of them, as far as there are tiles across; without this term 1084
// tokens of 208 x 15744 in 4 bits took 36 us by tiles of 32 tokens and 32 features, 22 by larger
// ones).
struct Variant {
  int rows, tokens, threads, waves, columns, lds, blocks;
  bool splits;
  int resident;
  float c[12];
  Launch launch[2];  // plain and gated
};

constexpr int CUS = 256;
constexpr int SPLITS[] = {1, 2, 3, 4, 6, 8};  // (those of sum_splits)
constexpr int SPLIT_COLUMNS = 512;           // at least, of a split of a tile
constexpr int64_t MOST_GRID_Y = 65535;

struct Plan {
  const Variant* variant;
  Grid grid;
  int splits;
  int64_t bytes;  // of partial sums
};

// The least estimate among those whose partial sums fit into `room` bytes and whose threads a
// launch can have (no variant, if there is none: near 2^39 outputs).
template <int COUNT>
Plan choose(const Variant (&variants)[COUNT], bool gated, int m, int n, int k, int64_t weight_bytes,
            int64_t room) {
  Plan best{nullptr, {0, 0}, 1, 0};
  float least = 0.f;
  for (const Variant& v : variants) {
    if (!v.launch[gated]) continue;
    const int features = gated ? v.rows / 2 : v.rows;
    const Grid g{((int64_t)m + v.tokens - 1) / v.tokens, ((int64_t)n + features - 1) / features};
    if (g.down > MOST_GRID_Y && !v.splits) continue;
    const int64_t tiles = g.down * g.across;
    const int64_t bytes = (int64_t)v.rows * std::max(v.tokens, 16) * 4 * tiles;
    const float* c = v.c;
    const float fixed = c[0] + c[6] * 1e-6f * (float)weight_bytes;
    const int steps = v.waves ? (k + v.columns - 1) / v.columns : 0;
    for (int splits : SPLITS) {
      if (tiles * splits * v.threads > dlfp::MOST_THREADS) break;
      if (splits > 1 && (!v.splits || splits * bytes > room ||
                         (v.waves ? splits * v.waves > steps : splits * SPLIT_COLUMNS > k)))
        break;
      if (v.blocks &&
          v.lds + v.blocks * (int64_t)dlfp::exps_bytes(k, splits, v.columns) > 160 * 1024)
        continue;
      const float u = (float)(tiles * splits) / CUS;
      const float r = (float)((tiles * splits + CUS - 1) / CUS);
      const int share = splits * v.waves;
      const float s =
          v.waves ? (float)((steps + share - 1) / share) : (float)k / 64 / (float)splits;
      float t = fixed + c[1] * s + (c[2] + c[3] * s) * u + (c[4] + c[5] * s) * r;
      if (v.resident) {
        const int64_t most = (int64_t)CUS * v.resident;
        t += (c[7] + c[8] * s) * (float)((tiles * splits + most - 1) / most);
      }
      if (splits > 1) t += c[9] + c[10] * 1e-6f * (float)(splits * bytes);
      if (v.waves) t += c[11] * 2e-6f * (float)((int64_t)m * k * std::min<int64_t>(8, g.across));
      if (best.variant && t >= least) continue;
      least = t;
      best = Plan{&v, g, splits, splits > 1 ? splits * bytes : 0};
    }
  }
  return best;
}

// Weights of one tile of tokens are read once; from here on they are read past the caches, which
// would not keep them until the next call anyway: 2 x 12288 x 4096 in bf16 (201 MB) 34.6 -> 31.6 us
// with 8 tokens, 42.3 -> 39.9 with 64; 2 x 25600 x 5120 in 4 bits (139 MB) 31.2 -> 29.8 with 8.
// Below, the 256 MB cache may have them from the last call (12288 x 4096 in 4 bits, 27 MB of 320 in
// turn: 12.9 -> 14.8 us past it).
constexpr int64_t STREAM_BYTES = 64 << 20;

bool past_caches(const Plan& p, int64_t weight_bytes) {
  return p.grid.down == 1 && weight_bytes >= STREAM_BYTES;
}

template <int COUNT>
dlfp::Form form_of(const Variant (&variants)[COUNT], bool gated, int m, int n, int k,
                   int64_t weight_bytes, int64_t room) {
  const Plan p = choose(variants, gated, m, n, k, weight_bytes, room);
  if (!p.variant) return dlfp::Form{-1, 0, 0, 1, 0, 0};
  return dlfp::Form{(int)(p.variant - variants), p.variant->rows,
                    p.variant->tokens,           p.splits,
                    past_caches(p, weight_bytes), p.bytes};
}

template <int COUNT>
int launch_best(const Variant (&variants)[COUNT], bool gated, dlfp::ProjectionArgs& a,
                int64_t weight_bytes, void* workspace, size_t bytes, hipStream_t stream) {
  const int64_t room = workspace ? (int64_t)std::min<size_t>(bytes, dlfp::MOST_PARTS) : 0;
  const Plan p = choose(variants, gated, a.m, a.n, a.k, weight_bytes, room);
  if (!p.variant) return DLFP_ERANGE;
  a.stream = past_caches(p, weight_bytes);
  return p.variant->launch[gated](a, p.grid, dlfp::Split{static_cast<float*>(workspace), p.splits},
                                  stream);
}

}  // namespace
