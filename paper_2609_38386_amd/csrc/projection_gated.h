// Gated projections with bf16 weights: the kernel of projection_few.h whose steps are 128 columns
// deep, and tile_kernel of projection_tiles.h with K over workgroups and with loops whose slots
// and conditions are settled when they are compiled (4096 tokens of 2 x 12288 x 4096: 671-684 us
// as GATED tile_kernel, 650-669 this way, 1.23-1.27 PFLOP/s, the matrix cores 65% busy: bound by
// what the power limit leaves of them; 64 tokens: 201 MB in 40-43 us, bound by HBM).
#pragma once

#include <type_traits>

#include "projection_sums.h"

namespace {

// ---------------------------------------------------------------- few tokens

constexpr int BSTEP = 128;  // columns of a step

template <int BLOCKS, int TOKENS, int WAVES, int DEPTH>
struct GatedFewShape {
  static constexpr int TB = TOKENS < 16 ? 1 : TOKENS / 16;
  static constexpr int WC = 4 * BLOCKS;                   // copies: of weights
  static constexpr int XC = TOKENS < 4 ? 1 : TOKENS / 4;  // of tokens
  static constexpr int SLOT = BLOCKS * 4096 + TOKENS * 256;
  static constexpr int RING = DEPTH * SLOT, RESULT = BLOCKS * TB * 1024;
  static constexpr int LDS = WAVES * (RING > RESULT ? RING : RESULT);
};

template <int BLOCKS, int TOKENS, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void gated_few_kernel(dlfp::ProjectionArgs a,
                                                               dlfp::Split split) {
  using Shape = GatedFewShape<BLOCKS, TOKENS, WAVES, DEPTH>;
  constexpr int TB = Shape::TB, WC = Shape::WC, XC = Shape::XC, L = WC + XC, SLOT = Shape::SLOT;
  static_assert(Shape::LDS <= LDS_MAX, "LDS");
  __shared__ __attribute__((aligned(16))) char smem[Shape::LDS];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  constexpr int FEATURES = 8 * BLOCKS;
  const Unit own = unit_of<FEATURES, TOKENS>(a, split, (a.k + BSTEP - 1) / BSTEP);
  const int n0 = own.n0, m0 = own.m0;
  const int first = own.from + wave, count = (own.to - first + WAVES - 1) / WAVES;

  // Copies: row 4 c + lane / 16 of 256 bytes, the 16 that belong at position lane % 16.
  uint32_t woff[4], xoff[XC];
  int wg[4], xg[XC];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int r = 4 * c + (lane >> 4);
    wg[c] = (lane & 15) ^ r;
    woff[c] = (uint32_t)(r * a.k * 2 + 16 * wg[c]);
  }
#pragma unroll
  for (int c = 0; c < XC; ++c) {
    const int r = 4 * c + (lane >> 4);
    xg[c] = (lane & 15) ^ (r & (TOKENS < 16 ? TOKENS - 1 : 15));
    xoff[c] = (uint32_t)(min(r, a.m - 1 - m0) * (int)a.ldx * 2 + 16 * xg[c]);
  }
  const char* wbase[BLOCKS];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
    wbase[b] = static_cast<const char*>(a.weights[b & 1]) +
               (int64_t)min(n0 + 16 * (b >> 1), a.n - 16) * a.k * 2;
  const char* xbase = reinterpret_cast<const char*>(a.x + (int64_t)m0 * a.ldx);
  char* ring = smem + wave * Shape::RING;
  const uint32_t lds0 = lds_addr(ring);
  auto issue = [&](auto inside, int t, int slot) {
    const int s = first + WAVES * t;
    const bool whole = inside.value || (s + 1) * BSTEP <= a.k;  // else its first half twice
    const uint32_t d = lds0 + slot * SLOT;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t off = whole || wg[c] < 8 ? woff[c] : woff[c] - 128;
        const uint32_t to = d + b * 4096 + c * 1024;
        if (a.stream)
          lds_stream16(wbase[b] + (int64_t)s * (2 * BSTEP), off, to);
        else
          lds_copy16(wbase[b] + (int64_t)s * (2 * BSTEP), off, to);
      }
#pragma unroll
    for (int c = 0; c < XC; ++c)
      if (TOKENS >= 4 || lane < 16 * TOKENS)
        lds_copy16(xbase + (int64_t)s * (2 * BSTEP), whole || xg[c] < 8 ? xoff[c] : xoff[c] - 128,
                   d + BLOCKS * 4096 + c * 1024);
  };
#pragma unroll
  for (int t = 0; t < DEPTH; ++t)
    if (t < count) issue(std::false_type{}, t, t);

  f32x4_t acc[BLOCKS][TB];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int u = 0; u < TB; ++u) acc[b][u] = f32x4_t{};
  const int lr = lane & 15, quad = lane >> 4, tr = lr & (TOKENS - 1);
  int slot = 0;
  // `inside`: the steps that a step looks ahead to are there, and it and they are whole ones.
  auto step = [&](auto inside, int t) {
    if constexpr (decltype(inside)::value)
      wait_copies<(DEPTH - 1) * L>();
    else
      wait_stages<DEPTH - 1, L, false>(count - 1 - t);
    const char* p = ring + slot * SLOT;
    bf16x8_t w[BLOCKS][4], xf[TB][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b)
        w[b][i] = *reinterpret_cast<const bf16x8_t*>(p + b * 4096 + lr * 256 +
                                                     (((4 * i + quad) ^ lr) << 4));
#pragma unroll
      for (int u = 0; u < TB; ++u)
        xf[u][i] = *reinterpret_cast<const bf16x8_t*>(p + BLOCKS * 4096 + (16 * u + tr) * 256 +
                                                      (((4 * i + quad) ^ tr) << 4));
    }
    wait_lds();  // the slot's reads have returned before it is refilled
    if (inside.value || t + DEPTH < count) issue(inside, t + DEPTH, slot);
    const bool whole = inside.value || (first + WAVES * t + 1) * BSTEP <= a.k;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < 2 || whole)  // (the second half of a last step of 64 columns is not there)
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
          for (int u = 0; u < TB; ++u)
            acc[b][u] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[b][i], xf[u][i], acc[b][u], 0, 0, 0);
    slot = slot + 1 == DEPTH ? 0 : slot + 1;
  };
  int t = 0;
  for (; t + DEPTH + 1 < count; ++t) step(std::true_type{}, t);
  for (; t < count; ++t) step(std::false_type{}, t);
  store_few<BLOCKS, TOKENS, WAVES, true>(a, split, acc, smem, tid, wave, own);
}

// ---------------------------------------------------------------- tiles

template <int TN, int TM, int WN, int WM, int STAGES>
__global__ __launch_bounds__(64 * WN * WM, 2) void gated_tile_kernel(dlfp::ProjectionArgs a,
                                                                     int gm, int gn,
                                                                     dlfp::Split split) {
  constexpr int WAVES = WN * WM, BN = TN / WN / 32, BM = TM / WM / 32, KK = KSTEP / 16;
  constexpr int NL = TN / (COPY_ROWS * WAVES), ML = TM / (COPY_ROWS * WAVES), L = NL + ML;
  static_assert(NL * COPY_ROWS * WAVES == TN && ML * COPY_ROWS * WAVES == TM, "copies");
  static_assert(WAVES % 4 == 0, "the copies of a wave are of one weight");
  constexpr int STAGE = (TN + TM) * ROW_BYTES;
  static_assert(STAGES * STAGE <= LDS_MAX, "LDS");
  __shared__ __attribute__((aligned(16))) char smem[STAGES * STAGE];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  // Units (tiles of a split, split after split) of an XCD as tiles in tile_kernel.
  const int tiles = gm * gn, units = tiles * split.splits, xcd = blockIdx.x & 7;
  const int unit = xcd * (units >> 3) + min(xcd, units & 7) + (blockIdx.x >> 3);
  const int part = unit / tiles, t = unit - part * tiles;
  constexpr int BAND = 8;
  const int first = t / (BAND * gn) * BAND, h = min(BAND, gm - first), in = t - first * gn;
  const int n0 = (in / h) * (TN / 2), m0 = (first + in % h) * TM;
  const int from = (int)((int64_t)(a.k / KSTEP) * part / split.splits);
  const int steps = (int)((int64_t)(a.k / KSTEP) * (part + 1) / split.splits) - from;

  const char* wbase = weight_rows(a, copy_weights<true>(wave), n0) + (int64_t)from * ROW_BYTES;
  const char* xbase = reinterpret_cast<const char*>(a.x + (int64_t)m0 * a.ldx) +
                      (int64_t)from * ROW_BYTES;
  uint32_t woff[NL], xoff[ML];
  weight_offsets<true>(woff, lane, a.k, a.n - 1 - n0, [&](int i) { return i * WAVES + wave; });
  copy_offsets(xoff, lane, (int)a.ldx, a.m - 1 - m0,
               [&](int i) { return COPY_ROWS * (i * WAVES + wave); });
  const uint32_t lds0 = lds_addr(smem) + wave * 1024;
  auto issue = [&](int ks, int slot) {
    const int64_t ko = (int64_t)ks * ROW_BYTES;
    const uint32_t d = lds0 + slot * STAGE;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      if (a.stream)
        lds_stream16(wbase + ko, woff[j], d + j * WAVES * 1024);
      else
        lds_copy16(wbase + ko, woff[j], d + j * WAVES * 1024);
    }
#pragma unroll
    for (int j = 0; j < ML; ++j)
      lds_copy16(xbase + ko, xoff[j], d + TN * ROW_BYTES + j * WAVES * 1024);
  };

  f32x16_t acc[BN][BM];
#pragma unroll
  for (int i = 0; i < BN; ++i)
#pragma unroll
    for (int j = 0; j < BM; ++j) acc[i][j] = f32x16_t{};
  const int lr = lane & 31, lh = lane >> 5, wn = wave / WM, wm = wave % WM;
  const char* wl = smem + (wn * BN * 32 + lr) * ROW_BYTES;
  const char* xl = smem + (TN + wm * BM * 32 + lr) * ROW_BYTES;
  bf16x8_t wf[2][BN], xf[2][BM];
  auto read = [&](int slot, int kk, int set) {
    const int c = slot * STAGE + (((2 * kk + lh) ^ swz(lr)) << 4);
#pragma unroll
    for (int q = 0; q < BN; ++q)
      wf[set][q] = *reinterpret_cast<const bf16x8_t*>(wl + 32 * q * ROW_BYTES + c);
#pragma unroll
    for (int q = 0; q < BM; ++q)
      xf[set][q] = *reinterpret_cast<const bf16x8_t*>(xl + 32 * q * ROW_BYTES + c);
  };
  auto multiply = [&](int set) {
#pragma unroll
    for (int q = 0; q < BN; ++q)
#pragma unroll
      for (int u = 0; u < BM; ++u)
        acc[q][u] =
            __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[set][q], xf[set][u], acc[q][u], 0, 0, 0);
  };

#pragma unroll
  for (int s = 0; s < STAGES; ++s)
    if (s < steps) issue(s, s);
  wait_stages<STAGES - 1, L, true>(steps - 1);
  read(0, 0, 0);
  // Step ks, in slot SLOT.  `inside`: all steps that it looks ahead to are there.
  auto step = [&](auto inside, auto slot_c, int ks) {
    constexpr bool INSIDE = decltype(inside)::value;
    constexpr int SLOT = decltype(slot_c)::value, NEXT = (SLOT + 1) % STAGES;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (kk + 1 < KK) {
        read(SLOT, kk + 1, (kk + 1) & 1);
      } else if (INSIDE || ks + 1 < steps) {
        // Stage ks + 1 has landed and no wave reads stage ks any more.
        if constexpr (INSIDE)
          wait_copies_barrier<(STAGES - 2) * L>();
        else
          wait_stages<STAGES - 2, L, true>(steps - 2 - ks);
        read(NEXT, 0, 0);
        if (INSIDE || ks + STAGES < steps) issue(ks + STAGES, SLOT);
      }
      multiply(kk & 1);
    }
  };
  auto round = [&](auto inside, int ks) {
    constexpr bool INSIDE = decltype(inside)::value;
    step(inside, std::integral_constant<int, 0>{}, ks);
    if (INSIDE || ks + 1 < steps) step(inside, std::integral_constant<int, 1 % STAGES>{}, ks + 1);
    if constexpr (STAGES > 2) {
      if (INSIDE || ks + 2 < steps) step(inside, std::integral_constant<int, 2 % STAGES>{}, ks + 2);
    }
    if constexpr (STAGES > 3) {
      if (INSIDE || ks + 3 < steps) step(inside, std::integral_constant<int, 3 % STAGES>{}, ks + 3);
    }
  };
  static_assert(STAGES >= 2 && STAGES <= 4, "slots of a round");
  int ks = 0;
  for (; ks + 2 * STAGES <= steps; ks += STAGES) round(std::true_type{}, ks);
  for (; ks < steps; ks += STAGES) round(std::false_type{}, ks);

  if (split.splits > 1) return store_parts(split, acc, (int64_t)unit * WAVES + wave, lane);
  constexpr int SLICE = STAGES * STAGE / WAVES / 16 * 16;
  wait_copies_barrier<0>();
  store_tile<BN, BM, SLICE, true>(a, acc, smem + wave * SLICE, lane, n0 + 16 * wn * BN,
                                  m0 + 32 * wm * BM);
}

}  // namespace
