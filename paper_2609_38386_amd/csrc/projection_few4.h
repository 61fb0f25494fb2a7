// Projections of few tokens with 4-bit weights: the kernel of projection_few.h whose steps are
// 256 columns deep.  Of a block, lane l takes row l % 16 and, of half h of a step, group
// 4 h + l / 16: 16 bytes of codes that are the operands of four products; which columns a
// product takes is free as long as both operands agree.  The exponents of the block's rows are
// one contiguous piece of memory, copied whole before the first step.
#pragma once

#include "projection_few.h"

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
  auto issue = [&](auto inside, int t, int slot) {
    const int s = first + t;
    // Past the row's end the step's first group again.
    const bool whole = inside.value || 8 * s + 8 <= groups;
    const uint32_t d = lds0 + slot * SLOT;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t off = whole || 8 * s + wg[c] < groups ? woff[c] : woff[c] - 16 * wg[c];
        const uint32_t to = d + b * 2048 + c * 1024;
        if (a.stream)
          lds_stream16(wbase[b] + (int64_t)s * 128, off, to);
        else
          lds_copy16(wbase[b] + (int64_t)s * 128, off, to);
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
    if (t < count) issue(std::false_type{}, t, t);

  f32x4_t acc[BLOCKS][TB];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int u = 0; u < TB; ++u) acc[b][u] = f32x4_t{};
  const int lr = lane & 15, quad = lane >> 4, tr = lr & (TOKENS - 1);
  const char* ex = smem + Shape::RINGS + lr * groups + quad;
  wait_stages<DEPTH, L, true>(count);  // the exponents of every wavefront are there
  int slot = 0;
  // `inside`: the steps that a step looks ahead to are there, and it and they are whole ones.
  auto step = [&](auto inside, int t) {
    if constexpr (decltype(inside)::value)
      wait_copies<(DEPTH - 1) * L>();
    else
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
    if (inside.value || t + DEPTH < count) issue(inside, t + DEPTH, slot);
    if (!inside.value && 8 * (first + t) + 8 > groups) {  // past the end of the rows: zeros
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
  };
  int t = 0;
  for (; t + DEPTH + 1 < count; ++t) step(std::true_type{}, t);
  for (; t < count; ++t) step(std::false_type{}, t);

  store_few<BLOCKS, TOKENS, WAVES, GATED>(a, split, acc, smem, tid, wave, unit, part, n0, m0);
}

}  // namespace
