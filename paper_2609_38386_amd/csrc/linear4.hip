// Projections with 4-bit weights: dlfp_linear_w4, dlfp_gated_linear_w4.  The kernels are those
// of projection_few4.h and projection_tiles4.h, and a plain one for rows that are far apart.
#include <algorithm>

#include "dlfp_ffn.h"
#include "projection_few4.h"
#include "projection_tiles4.h"

namespace {

// ---------------------------------------------------------------- far rows

// Rows of x or of weights 2^22 elements and more apart: 16 features and 16 tokens a workgroup,
// operands straight from memory with 64-bit addresses, K over eight wavefronts in steps of 128
// columns.  (The other kernels' copies have 32-bit offsets from a tile's first row.)
constexpr int FAR_STRIDE = 1 << 22, FAR_WAVES = 8, FAR_STEP = 128;

template <bool GATED>
__global__ __launch_bounds__(64 * FAR_WAVES) void far4_kernel(dlfp::ProjectionArgs a) {
  constexpr int B = GATED ? 2 : 1;
  __shared__ f32x4_t sums[FAR_WAVES][B][64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, lr = lane & 15, quad = lane >> 4;
  const uint32_t gn = (uint32_t)a.n / 16;
  const int n0 = (int)(blockIdx.x % gn) * 16, m0 = (int)(blockIdx.x / gn) * 16;
  const uint16_t* x = a.x + (int64_t)min(m0 + lr, a.m - 1) * a.ldx;
  f32x4_t acc[B] = {};
  for (int k0 = FAR_STEP * wave; k0 < a.k; k0 += FAR_STEP * FAR_WAVES) {
    // Of a last step of 64 columns half of the lanes' columns are past the row: zeros.
    const int c = k0 + 32 * quad;
    const bool in = c < a.k;
    bf16x8_t xf[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
      xf[t] = in ? *reinterpret_cast<const bf16x8_t*>(x + c + 8 * t) : bf16x8_t{};
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int64_t row = n0 + lr;
      const char* codes = static_cast<const char*>(a.weights[b]) + row * (a.k >> 1);
      const u32x4_t w = in ? *reinterpret_cast<const u32x4_t*>(codes + (c >> 1)) : u32x4_t{};
      const float scale = scale_of(in ? a.exps[b][row * (a.k >> 5) + (c >> 5)] : 0);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w[t], scale), xf[t], acc[b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int b = 0; b < B; ++b) sums[wave][b][lane] = acc[b];
  __syncthreads();
  if (wave) return;
  f32x4_t v = sums[0][0][lane], up = sums[0][B - 1][lane];
#pragma unroll
  for (int w = 1; w < FAR_WAVES; ++w) {
    v += sums[w][0][lane];
    up += sums[w][B - 1][lane];
  }
  if constexpr (GATED) v = gated4(v, up, a.act);
  if (m0 + lr < a.m) store4(a, m0 + lr, n0 + 4 * quad, v);
}

template <bool GATED>
int launch_far(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  const int64_t blocks = (int64_t)(a.n / 16) * (((int64_t)a.m + 15) / 16);
  if (blocks * (64 * FAR_WAVES) >= (int64_t)1 << 32) return DLFP_ERANGE;
  far4_kernel<GATED><<<(uint32_t)blocks, 64 * FAR_WAVES, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

// ---------------------------------------------------------------- launches

// `down` x `across` tiles of tokens and features.
struct Grid {
  int64_t down, across;
};

template <bool GATED, int BLOCKS, int TOKENS, int WAVES, int DEPTH>
int launch_few(const dlfp::ProjectionArgs& a, Grid g, dlfp::Split split, hipStream_t stream) {
  if constexpr (GATED && BLOCKS % 2) {
    return DLFP_EUNSUPPORTED;
  } else {
    using Shape = FewShape<BLOCKS, TOKENS, WAVES, DEPTH>;
    const int64_t tiles = g.down * g.across;
    if (tiles * split.splits * (64 * WAVES) >= (int64_t)1 << 32) return DLFP_ERANGE;
    few4_kernel<BLOCKS, TOKENS, WAVES, DEPTH, GATED>
        <<<(uint32_t)(tiles * split.splits), 64 * WAVES, (size_t)Shape::lds(a.k), stream>>>(a,
                                                                                          split);
    if (split.splits > 1) {
      constexpr int UNITS = (GATED ? BLOCKS / 2 : BLOCKS) * Shape::TB;
      sum_few_kernel<BLOCKS, TOKENS, GATED><<<(uint32_t)(tiles * UNITS), 64, 0, stream>>>(
          a, (int)g.across, (int)tiles, split);
    }
    return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
  }
}

template <bool GATED, int TN, int TM, int WN, int WM, int DEPTH, int STAGES, bool WHOLE>
int launch_tile(const dlfp::ProjectionArgs& a, Grid g, dlfp::Split split, hipStream_t stream) {
  const int64_t tiles = g.down * g.across;
  if (tiles * split.splits * (64 * WN * WM) >= (int64_t)1 << 32) return DLFP_ERANGE;
  tile4_kernel<TN, TM, WN, WM, DEPTH, STAGES, GATED, WHOLE>
      <<<(uint32_t)(tiles * split.splits), 64 * WN * WM, 0, stream>>>(a, (int)g.down,
                                                                      (int)g.across, split);
  if (split.splits > 1) {
    constexpr int BLOCKS = TN * TM / 16 * (GATED ? 2 : 4) / 256;
    sum_tiles_kernel<TN, TM, WN, WM, GATED><<<(uint32_t)(tiles * BLOCKS), 256, 0, stream>>>(
        a, (int)g.down, (int)g.across, split);
  }
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

// ---------------------------------------------------------------- choice

typedef int (*Launch)(const dlfp::ProjectionArgs&, Grid, dlfp::Split, hipStream_t);

// A tile of `rows` rows of weights and `tokens` tokens.  Its time in microseconds, of u = units
// (tiles times splits) / 256 and s = K steps of a unit (of 64 columns; in few4_kernel of 256 of
// a wavefront):
//   start + step s + (unit + work s) u + (round + turn s) ceil(u)
//   + with splits: join + partial sums * (units' fp32 MB)
struct Variant {
  int rows, tokens;
  int waves;        // that share the K steps of a unit; 0: of tile4_kernel
  int rings, blocks;  // LDS of few4_kernel beside the exponents, and its blocks of 16 rows
  float start, step, unit, work, round, turn, join, part;
  Launch plain, gated;
};
#define FEW(B, T, W, D)                                                                       \
  16 * B, T, W, FewShape<B, T, W, D>::RINGS, B
#define FEW_LAUNCH(B, T, W, D) launch_few<false, B, T, W, D>, launch_few<true, B, T, W, D>
#define TILE(TN, TM) TN, TM, 0, 0, 0
#define TILE_LAUNCH(...) launch_tile<false, __VA_ARGS__>, launch_tile<true, __VA_ARGS__>
constexpr Variant VARIANTS[] = {
    {FEW(1, 2, 4, 2), 2.559f, 0.146f, 0.f, 0.103f, 0.f, 0.174f, 2.266f, 0.261f, FEW_LAUNCH(1, 2, 4, 2)},
    {FEW(2, 2, 4, 1), 2.677f, 0.215f, 0.f, 0.299f, 0.f, 0.238f, 2.37f, 0.406f, FEW_LAUNCH(2, 2, 4, 1)},
    {FEW(1, 4, 8, 2), 2.417f, 0.091f, 0.f, 0.26f, 0.276f, 0.36f, 2.103f, 0.593f, FEW_LAUNCH(1, 4, 8, 2)},
    {FEW(2, 4, 4, 2), 2.734f, 0.131f, 0.03f, 0.248f, 0.f, 0.363f, 2.287f, 0.727f, FEW_LAUNCH(2, 4, 4, 2)},
    {FEW(1, 8, 8, 2), 1.559f, 0.f, 0.f, 0.301f, 1.141f, 0.553f, 2.133f, 1.015f, FEW_LAUNCH(1, 8, 8, 2)},
    {FEW(2, 8, 4, 1), 2.744f, 0.291f, 0.f, 0.394f, 0.f, 0.22f, 2.391f, 0.332f, FEW_LAUNCH(2, 8, 4, 1)},
    {FEW(1, 16, 4, 1), 2.551f, 0.177f, 0.f, 0.249f, 0.f, 0.294f, 2.289f, 0.029f, FEW_LAUNCH(1, 16, 4, 1)},
    {FEW(2, 16, 4, 1), 2.753f, 0.27f, 0.f, 0.423f, 0.f, 0.37f, 2.317f, 0.701f, FEW_LAUNCH(2, 16, 4, 1)},
    {FEW(4, 16, 4, 1), 2.912f, 0.334f, 0.f, 0.828f, 0.f, 0.632f, 2.558f, 0.522f, FEW_LAUNCH(4, 16, 4, 1)},
    {FEW(2, 32, 2, 1), 2.678f, 0.42f, 0.021f, 0.13f, 0.313f, 0.396f, 2.639f, 0.193f, FEW_LAUNCH(2, 32, 2, 1)},
    {FEW(2, 32, 6, 1), 1.225f, 0.101f, 0.f, 0.598f, 1.725f, 1.117f, 2.738f, 0.338f, FEW_LAUNCH(2, 32, 6, 1)},
    {TILE(128, 32), 2.453f, 0.143f, 0.274f, 0.068f, 0.777f, 0.085f, 2.792f, 0.261f, TILE_LAUNCH(128, 32, 4, 1, 4, 3, true)},
    {TILE(128, 64), 2.922f, 0.294f, 0.708f, 0.131f, 0.269f, 0.06f, 2.599f, 0.254f, TILE_LAUNCH(128, 64, 4, 1, 2, 2, false)},
    {TILE(256, 64), 2.059f, 0.026f, 1.4f, 0.112f, 1.967f, 0.365f, 2.636f, 0.304f, TILE_LAUNCH(256, 64, 8, 1, 4, 3, true)},
    {TILE(256, 128), 2.222f, 0.f, 2.68f, 0.161f, 2.569f, 0.649f, 2.767f, 0.229f, TILE_LAUNCH(256, 128, 8, 1, 4, 3, false)},
    {TILE(256, 256), 3.128f, 0.f, 5.166f, 0.311f, 2.721f, 1.109f, 3.928f, 0.162f, TILE_LAUNCH(256, 256, 8, 1, 2, 2, false)},
};
#undef FEW
#undef FEW_LAUNCH
#undef TILE
#undef TILE_LAUNCH
constexpr int CUS = 256;
constexpr int SPLITS[] = {1, 2, 3, 4, 6, 8};
constexpr int64_t MOST_PARTS = 32 << 20;  // bytes of partial sums

struct Plan {
  const Variant* variant;
  Grid grid;
  int splits;
  int64_t bytes;  // of partial sums
};

// The variant and the number of splits whose estimated time is lowest, of those whose partial
// sums fit into `room` bytes.
Plan choose(bool gated, int m, int n, int k, int64_t room) {
  Plan best{nullptr, {0, 0}, 1, 0};
  float least = 0.f;
  const int steps = (k + FSTEP - 1) / FSTEP;
  for (const Variant& v : VARIANTS) {
    if (gated && v.rows < 32) continue;
    if (v.waves && v.rings + v.blocks * (((int64_t)k / 2 + 1023) / 1024 * 1024) > LDS_MAX) continue;
    const int features = gated ? v.rows / 2 : v.rows;
    const Grid g{((int64_t)m + v.tokens - 1) / v.tokens, ((int64_t)n + features - 1) / features};
    const int64_t tiles = g.down * g.across;
    const int64_t bytes = (int64_t)v.rows * std::max(v.tokens, 16) * 4 * tiles;
    for (int splits : SPLITS) {
      if (splits > 1 && (splits * bytes > room || splits * std::max(v.waves, 2) > steps)) break;
      const float u = (float)(tiles * splits) / CUS;
      const float r = (float)((tiles * splits + CUS - 1) / CUS);
      const int per = splits * v.waves;
      const float s = v.waves ? (float)((steps + per - 1) / per) : (float)k / KSTEP / (float)splits;
      float t = v.start + v.step * s + (v.unit + v.work * s) * u + (v.round + v.turn * s) * r;
      if (splits > 1) t += v.join + v.part * 1e-6f * (float)(splits * bytes);
      if (best.variant && t >= least) continue;
      least = t;
      best = Plan{&v, g, splits, splits > 1 ? splits * bytes : 0};
    }
  }
  return best;
}

template <bool GATED>
int launch(const dlfp::ProjectionArgs& a, void* workspace, size_t bytes, hipStream_t stream) {
  (void)hipGetLastError();
  if (std::max<int64_t>(a.ldx, a.k) >= FAR_STRIDE) return launch_far<GATED>(a, stream);
  const int64_t room = workspace ? (int64_t)std::min<size_t>(bytes, MOST_PARTS) : 0;
  const Plan p = choose(GATED, a.m, a.n, a.k, room);
  const dlfp::Split split{static_cast<float*>(workspace), p.splits};
  return (GATED ? p.variant->gated : p.variant->plain)(a, p.grid, split, stream);
}

}  // namespace

namespace dlfp {

int check_projection(ProjectionArgs& a, bool gated, bool codes, int32_t out_dtype,
                     const void* workspace) {
  if (a.m < 0 || a.n <= 0 || a.k <= 0) return DLFP_EINVAL;
  if (out_dtype != 0 && out_dtype != 1) return DLFP_EINVAL;
  if (gated && a.act != DLFP_SILU && a.act != DLFP_GELU) return DLFP_EINVAL;
  if (a.n % 16 || a.k % 64) return DLFP_EUNSUPPORTED;
  if (a.ldx < a.k || a.ldo < a.n || a.ldx % 8 || a.ldo % 4) return DLFP_EINVAL;
  if (a.m == 0) return DLFP_OK;
  const auto aligned = [](const void* p, uintptr_t to) {
    return p && reinterpret_cast<uintptr_t>(p) % to == 0;
  };
  if (!aligned(a.x, 16) || !aligned(a.out, out_dtype ? 16 : 8)) return DLFP_EINVAL;
  if (workspace && !aligned(workspace, 16)) return DLFP_EINVAL;
  for (int i = 0; i < (gated ? 2 : 1); ++i) {
    if (!aligned(a.weights[i], 16)) return DLFP_EINVAL;
    if (codes && !aligned(a.exps[i], 16)) return DLFP_EINVAL;
  }
  a.wide = aligned(a.out, 16) && a.ldo % 8 == 0;
  return DLFP_OK;
}

}  // namespace dlfp

extern "C" int dlfp_linear_w4(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                              const void* codes, const void* exps, void* out, int64_t ldo,
                              int32_t out_dtype, void* workspace, size_t workspace_bytes,
                              hipStream_t stream) {
  dlfp::ProjectionArgs a{static_cast<const uint16_t*>(x),
                         {codes, nullptr},
                         {static_cast<const uint8_t*>(exps), nullptr},
                         out, ldx, ldo, m, n, k, 0, out_dtype, 0};
  const int st = dlfp::check_projection(a, false, true, out_dtype, workspace);
  return st != DLFP_OK || m == 0 ? st : launch<false>(a, workspace, workspace_bytes, stream);
}

extern "C" int dlfp_gated_linear_w4(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                                    const void* gate_codes, const void* gate_exps,
                                    const void* up_codes, const void* up_exps, int32_t activation,
                                    void* out, int64_t ldo, int32_t out_dtype, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream) {
  dlfp::ProjectionArgs a{
      static_cast<const uint16_t*>(x),
      {gate_codes, up_codes},
      {static_cast<const uint8_t*>(gate_exps), static_cast<const uint8_t*>(up_exps)},
      out, ldx, ldo, m, n, k, activation, out_dtype, 0};
  const int st = dlfp::check_projection(a, true, true, out_dtype, workspace);
  return st != DLFP_OK || m == 0 ? st : launch<true>(a, workspace, workspace_bytes, stream);
}

extern "C" int64_t dlfp_projection_workspace(int32_t kind, int32_t m, int32_t n, int32_t k) {
  if (m <= 0 || n <= 0 || k <= 0 || n % 16 || k % 64 || k >= FAR_STRIDE) return 0;
  if (kind == DLFP_LINEAR_W4 || kind == DLFP_GATED_LINEAR_W4)
    return choose(kind == DLFP_GATED_LINEAR_W4, m, n, k, MOST_PARTS).bytes;
  return 0;
}
