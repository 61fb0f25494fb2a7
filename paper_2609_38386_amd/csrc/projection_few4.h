// Projections of few tokens with 4-bit weights: codes, exponents and tokens through LDS, by
// copies of whole row segments, into v_mfma_f32_16x16x32_bf16 as out^T = W x^T.
//
// A workgroup takes BLOCKS blocks of 16 rows of weights (gated: rows of the gate and of the up
// in turn) and TOKENS tokens.  Its wavefronts split K in steps of 256 columns, each through a
// ring of its own without barriers, and their results are added through LDS, in wavefront
// order.  Of a block, lane l takes row l % 16 and, of half h of a step, group 4 h + l / 16:
// 16 bytes of codes that are the operands of four products; which columns a product takes is
// free as long as both operands agree.  The exponents of the block's rows are one contiguous
// piece of memory, copied whole before the first step.
#pragma once

#include "projection_tiles4.h"

namespace {

constexpr int FSTEP = 256;  // columns of a step

template <int BLOCKS, int TOKENS, int WAVES, int DEPTH>
struct FewShape {
  static constexpr int TB = TOKENS < 16 ? 1 : TOKENS / 16;           // token blocks
  static constexpr int WC = 2 * BLOCKS;                              // copies: of weights
  static constexpr int XC = TOKENS < 2 ? 1 : TOKENS / 2;             // of tokens
  static constexpr int SLOT = BLOCKS * 2048 + TOKENS * 512;
  static constexpr int RING = DEPTH * SLOT, RESULT = BLOCKS * TB * 1024;
  static constexpr int RINGS = WAVES * (RING > RESULT ? RING : RESULT);
  // LDS of a launch: the rings, then each block's exponents in whole copies.
  static int64_t exps(int k) { return ((int64_t)k / 2 + 1023) / 1024 * 1024; }
  static int64_t lds(int k) { return RINGS + BLOCKS * exps(k); }
};

template <int BLOCKS, int TOKENS, int WAVES, int DEPTH, bool GATED>
__global__ __launch_bounds__(64 * WAVES) void few4_kernel(dlfp::ProjectionArgs a,
                                                                dlfp::Split split) {
  using Shape = FewShape<BLOCKS, TOKENS, WAVES, DEPTH>;
  constexpr int TB = Shape::TB, WC = Shape::WC, XC = Shape::XC, L = WC + XC, SLOT = Shape::SLOT;
  extern __shared__ __attribute__((aligned(16))) char few_lds[];
  char* smem = few_lds;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  constexpr int FEATURES = 16 * (GATED ? BLOCKS / 2 : BLOCKS);
  const uint32_t gn = (uint32_t)(a.n + FEATURES - 1) / FEATURES;
  const uint32_t unit = blockIdx.x / split.splits, part = blockIdx.x - unit * split.splits;
  const int n0 = (int)(unit % gn) * FEATURES, m0 = (int)(unit / gn) * TOKENS;
  const int groups = a.k >> 5, steps = (a.k + FSTEP - 1) / FSTEP;
  const int64_t shares = (int64_t)WAVES * split.splits, share = (int64_t)WAVES * part + wave;
  const int first = (int)(steps * share / shares);
  const int count = (int)(steps * (share + 1) / shares) - first;
  // First row of block b in its weights: past the end, the last 16 again.
  auto row0 = [&](int b) { return min(n0 + 16 * (GATED ? b >> 1 : b), a.n - 16); };

  // Copies of weights: rows 8 c + lane / 8, the group that belongs at position lane % 8; of
  // tokens: row 2 c + lane / 32, the 16 bytes that belong at position lane % 32.
  uint32_t woff[2], xoff[XC];
  int wg[2], xg[XC];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int r = 8 * c + (lane >> 3);
    wg[c] = (lane & 7) ^ swz(r);
    woff[c] = (uint32_t)(r * (a.k >> 1) + 16 * wg[c]);
  }
#pragma unroll
  for (int c = 0; c < XC; ++c) {
    const int r = 2 * c + (lane >> 5);
    xg[c] = (lane & 31) ^ (r & 15);
    xoff[c] = (uint32_t)(min(r, a.m - 1 - m0) * (int)a.ldx * 2 + 16 * xg[c]);
  }
  const char* wbase[BLOCKS];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
    wbase[b] = static_cast<const char*>(a.weights[GATED ? b & 1 : 0]) +
               (int64_t)row0(b) * (a.k >> 1);
  const char* xbase = reinterpret_cast<const char*>(a.x + (int64_t)m0 * a.ldx);
  char* ring = smem + wave * Shape::RING;
  const uint32_t lds0 = lds_addr(ring);
  auto issue = [&](int t, int slot) {
    const int s = first + t;
    const bool whole = 8 * s + 8 <= groups;  // else past the row's end the step's first again
    const uint32_t d = lds0 + slot * SLOT;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t off = whole || 8 * s + wg[c] < groups ? woff[c] : woff[c] - 16 * wg[c];
        lds_copy16(wbase[b] + (int64_t)s * 128, off, d + b * 2048 + c * 1024);
      }
#pragma unroll
    for (int c = 0; c < XC; ++c)
      if (TOKENS >= 2 || lane < 32) {
        const uint32_t off = whole || 8 * s + (xg[c] >> 2) < groups ? xoff[c] : xoff[c] - 16 * xg[c];
        lds_copy16(xbase + (int64_t)s * (2 * FSTEP), off, d + BLOCKS * 2048 + c * 1024);
      }
  };

  // Exponents: 16 rows of groups bytes are one piece of k / 2 bytes; the copies of a block are
  // dealt to the wavefronts.
  const int epieces = ((a.k >> 1) + 1023) / 1024, eblock = epieces * 1024;
  const uint32_t elds = lds_addr(smem) + Shape::RINGS;
  for (int i = wave; i < BLOCKS * epieces; i += WAVES) {
    const int b = i / epieces, p = i - b * epieces;
    const char* src = reinterpret_cast<const char*>(a.exps[GATED ? b & 1 : 0]) +
                      (int64_t)row0(b) * groups;
    lds_copy16(src, (uint32_t)min(p * 1024 + lane * 16, (a.k >> 1) - 16), elds + i * 1024);
  }
#pragma unroll
  for (int t = 0; t < DEPTH; ++t)
    if (t < count) issue(t, t);

  f32x4_t acc[BLOCKS][TB];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int u = 0; u < TB; ++u) acc[b][u] = f32x4_t{};
  const int lr = lane & 15, quad = lane >> 4, tr = lr & (TOKENS - 1);
  const char* ex = smem + Shape::RINGS + lr * groups + quad;
  wait_stages<DEPTH, L, true>(count);  // the exponents of every wavefront are there
  int slot = 0;
  for (int t = 0; t < count; ++t) {
    wait_stages<DEPTH - 1, L, false>(count - 1 - t);
    const char* p = ring + slot * SLOT;
    u32x4_t codes[2][BLOCKS];
    bf16x8_t xf[2][TB][4];
    uint32_t e[2][BLOCKS];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) {
        codes[h][b] = *reinterpret_cast<const u32x4_t*>(
            p + b * 2048 + lr * 128 + (((4 * h + quad) ^ swz(lr)) << 4));
        e[h][b] = *reinterpret_cast<const uint8_t*>(ex + b * eblock + 8 * (first + t) + 4 * h);
      }
#pragma unroll
      for (int u = 0; u < TB; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          xf[h][u][i] = *reinterpret_cast<const bf16x8_t*>(
              p + BLOCKS * 2048 + (16 * u + tr) * 512 +
              (((16 * h + 4 * quad + i) ^ tr) << 4));
    }
    wait_lds();  // the slot's reads have returned before it is refilled
    if (t + DEPTH < count) issue(t + DEPTH, slot);
    if (8 * (first + t) + 8 > groups) {  // past the end of the rows: zeros
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (8 * (first + t) + 4 * h + quad >= groups) {
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) codes[h][b] = u32x4_t{}, e[h][b] = 0;
#pragma unroll
          for (int u = 0; u < TB; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) xf[h][u][i] = bf16x8_t{};
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
          const bf16x8_t w = widen(codes[h][b][i], scale_of(e[h][b]));
#pragma unroll
          for (int u = 0; u < TB; ++u)
            acc[b][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, xf[h][u][i], acc[b][u], 0, 0, 0);
        }
    slot = slot + 1 == DEPTH ? 0 : slot + 1;
  }

  // Lane l holds features 4 (l / 16) .. + 3 of token l % 16 of a block: the waves' sum.
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
      f32x4_t* out = reinterpret_cast<f32x4_t*>(split.part) +
                     ((int64_t)part * (gridDim.x / split.splits) + unit) * (BLOCKS * TB * 64) + i;
      *out = v;
      if constexpr (GATED) out[OUT * TB * 64] = sum(2 * r + 1);
      continue;
    }
    if constexpr (GATED) v = gated4(v, sum(2 * r + 1), a.act);
    const int tok = 16 * u + (l & 15), m = m0 + tok, n = n0 + 16 * r + 4 * (l >> 4);
    if (tok < TOKENS && m < a.m && n < a.n) store4(a, m, n, v);
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
  f32x4_t v = p[0], up{};
  if constexpr (GATED) up = p[OUT * TB * 64];
  for (int s = 1; s < split.splits; ++s) {
    v += p[(int64_t)s * tiles * UNITS];
    if constexpr (GATED) up += p[(int64_t)s * tiles * UNITS + OUT * TB * 64];
  }
  if constexpr (GATED) v = gated4(v, up, a.act);
  store4(a, m, n, v);
}

}  // namespace
