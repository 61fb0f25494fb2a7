// Projections of few tokens with 4-bit weights: the kernel of projection_few.h whose steps are
// 128 or 256 columns deep.  Of a block, lane l takes row l % 16 and, of half h of a step, group
// 4 h + l / 16: 16 bytes of codes that are the operands of four products; which columns a
// product takes is free as long as both operands agree.
//
// The exponents of the block's rows are copied before the first step, one contiguous piece of
// memory; with K over workgroups, of each row the workgroup's part, which leaves the LDS to wider
// blocks (16 tokens of 5120 x 25600 in 3 parts, weights from HBM, 0.91 of the time).  As 4-byte pieces
// with each step they took a third of the copies' time (4096 x 12288, 1 token: 9.6 us against 8.4
// without any), and loaded into registers beside the copies they made every step wait for all copies
// in flight (16 tokens of 5120 x 25600: 22.9 against 21.2 us).  They are what limits k here: with more
// than the LDS holds, tiles are taken.
//
// Steps of 256 columns copy weights in rows of 128 bytes; steps of 128 columns (64-byte rows, which
// are copied at half the rate) let twice the wavefronts share the LDS, which pays where the
// tokens are most of the bytes (64 tokens of 12288 x 4096 17.6 -> 15.8 us).
#pragma once

#include "projection_few.h"

namespace {

constexpr int FHALF = 128;  // columns of a half: a step has one or two

template <int BLOCKS, int TOKENS, int WAVES, int DEPTH, int HALVES>
struct FewShape {
  static constexpr int TB = TOKENS < 16 ? 1 : TOKENS / 16;           // token blocks
  static constexpr int WC = HALVES * BLOCKS;                         // copies: of weights
  static constexpr int XC = (TOKENS * HALVES + 3) / 4;               // of tokens
  static constexpr int SLOT = HALVES * (BLOCKS * 1024 + TOKENS * 256);
  static constexpr int RING = DEPTH * SLOT, RESULT = BLOCKS * TB * 1024;
  static constexpr int RINGS = WAVES * (RING > RESULT ? RING : RESULT);
  // LDS of a launch: the rings, then each block's exponents.
  static int64_t lds(int k, int splits) {
    return RINGS + (int64_t)BLOCKS * dlfp::exps_bytes(k, splits, HALVES * FHALF);
  }
};

// Position of a row's 16 bytes of weights: rows of 128 bytes as in a tile, of 64 bytes spread over
// the banks by bits 2-3 of the row.
template <int HALVES>
__device__ __forceinline__ int few_swz(int row) {
  return HALVES == 2 ? swz(row) : (row >> 2) & 3;
}

template <int BLOCKS, int TOKENS, int WAVES, int DEPTH, int HALVES, bool GATED>
__global__ __launch_bounds__(64 * WAVES) void few4_kernel(dlfp::ProjectionArgs a,
                                                                dlfp::Split split) {
  using Shape = FewShape<BLOCKS, TOKENS, WAVES, DEPTH, HALVES>;
  constexpr int STEP = HALVES * FHALF, GROUPS = STEP / 32;  // of a step
  constexpr int TB = Shape::TB, WC = Shape::WC, XC = Shape::XC, L = WC + XC, SLOT = Shape::SLOT;
  extern __shared__ __attribute__((aligned(16))) char few_lds[];
  char* smem = few_lds;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  constexpr int FEATURES = 16 * (GATED ? BLOCKS / 2 : BLOCKS);
  const Unit own = unit_of<FEATURES, TOKENS>(a, split, (a.k + STEP - 1) / STEP);
  const int n0 = own.n0, m0 = own.m0, groups = a.k >> 5;
  const int first = own.from + wave, count = (own.to - first + WAVES - 1) / WAVES;
  // First row of block b in its weights: past the end, the last 16 again.
  auto row0 = [&](int b) { return min(n0 + 16 * (GATED ? b >> 1 : b), a.n - 16); };

  // Copies of weights: rows WROWS c + lane / GROUPS, the group that belongs at position
  // lane % GROUPS; of tokens: rows of 4 GROUPS pieces of 16 bytes.
  constexpr int WROWS = 64 / GROUPS, XPIECES = 4 * GROUPS, XROWS = 64 / XPIECES;
  uint32_t woff[HALVES], xoff[XC];
  int wg[HALVES], xg[XC];
#pragma unroll
  for (int c = 0; c < HALVES; ++c) {
    const int r = WROWS * c + lane / GROUPS;
    wg[c] = (lane % GROUPS) ^ few_swz<HALVES>(r);
    woff[c] = (uint32_t)(r * (a.k >> 1) + 16 * wg[c]);
  }
#pragma unroll
  for (int c = 0; c < XC; ++c) {
    const int r = XROWS * c + lane / XPIECES;
    xg[c] = (lane % XPIECES) ^ (r & (TOKENS < 16 ? TOKENS - 1 : 15));
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
    const int s = first + WAVES * t;
    // Past the row's end the step's first group again.
    const bool whole = inside.value || GROUPS * s + GROUPS <= groups;
    const uint32_t d = lds0 + slot * SLOT;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
      for (int c = 0; c < HALVES; ++c) {
        const uint32_t off =
            whole || GROUPS * s + wg[c] < groups ? woff[c] : woff[c] - 16 * wg[c];
        const uint32_t to = d + (b * HALVES + c) * 1024;
        const char* from = wbase[b] + (int64_t)s * (STEP / 2);
        // Rows of 64 bytes: past the caches each line would come from HBM twice (a call of 32
        // tokens of 5120 x 25600, weights from HBM: 28.1 against 25.9 us).
        if (HALVES == 2 && a.stream)
          lds_stream16(from, off, to);
        else
          lds_copy16(from, off, to);
      }
#pragma unroll
    for (int c = 0; c < XC; ++c)
      if (TOKENS >= XROWS || lane < XPIECES * TOKENS) {
        const uint32_t off =
            whole || GROUPS * s + (xg[c] >> 2) < groups ? xoff[c] : xoff[c] - 16 * xg[c];
        lds_copy16(xbase + (int64_t)s * (2 * STEP), off,
                   d + BLOCKS * HALVES * 1024 + c * 1024);
      }
  };

  // Exponents: 16 rows of groups bytes are one piece of k / 2 bytes; the copies of a block are
  // dealt to the wavefronts.  Of a split, a row's pieces of 16 bytes from the one on in which its
  // first group is.
  const int pitch = dlfp::exps_pitch(a.k, split.splits, STEP);
  const int eblock = dlfp::exps_bytes(a.k, split.splits, STEP), epieces = eblock / 1024;
  const int g0 = GROUPS * own.from;
  const uint32_t elds = lds_addr(smem) + Shape::RINGS;
  for (int i = wave; i < BLOCKS * epieces; i += WAVES) {
    const int b = i / epieces, p = i - b * epieces;
    const char* src = reinterpret_cast<const char*>(a.exps[GATED ? b & 1 : 0]) +
                      (int64_t)row0(b) * groups;
    int off = p * 1024 + lane * 16;
    if (split.splits > 1) {
      const int row = off / pitch;
      off = ((row * groups + g0) & ~15) + off - row * pitch;
    }
    lds_copy16(src, (uint32_t)min(off, (a.k >> 1) - 16), elds + i * 1024);
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
  const char* ex = smem + Shape::RINGS + lr * pitch + quad - g0;
  if (split.splits > 1) ex += (lr * groups + g0) & 15;
  wait_stages<DEPTH, L, true>(count);  // the exponents of every wavefront are there
  int slot = 0;
  // `inside`: the steps that a step looks ahead to are there, and it and they are whole ones.
  auto step = [&](auto inside, int t) {
    if constexpr (decltype(inside)::value)
      wait_copies<(DEPTH - 1) * L>();
    else
      wait_stages<DEPTH - 1, L, false>(count - 1 - t);
    const int g = GROUPS * (first + WAVES * t);
    const char* p = ring + slot * SLOT;
    u32x4_t codes[HALVES][BLOCKS];
    bf16x8_t xf[HALVES][TB][4];
    uint32_t e[HALVES][BLOCKS];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) {
        codes[h][b] = *reinterpret_cast<const u32x4_t*>(
            p + (b * 16 + lr) * (16 * GROUPS) + (((4 * h + quad) ^ few_swz<HALVES>(lr)) << 4));
        e[h][b] =
            *reinterpret_cast<const uint8_t*>(ex + b * eblock + g + 4 * h);
      }
#pragma unroll
      for (int u = 0; u < TB; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          xf[h][u][i] = *reinterpret_cast<const bf16x8_t*>(
              p + BLOCKS * HALVES * 1024 + (16 * u + tr) * (16 * XPIECES) +
              (((16 * h + 4 * quad + i) ^ tr) << 4));
    }
    wait_lds();  // the slot's reads have returned before it is refilled
    if (inside.value || t + DEPTH < count) issue(inside, t + DEPTH, slot);
    if (!inside.value && g + GROUPS > groups) {  // past the end of the rows: zeros
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
        if (g + 4 * h + quad >= groups) {
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) codes[h][b] = u32x4_t{}, e[h][b] = 0;
#pragma unroll
          for (int u = 0; u < TB; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) xf[h][u][i] = bf16x8_t{};
        }
    }
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
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

  store_few<BLOCKS, TOKENS, WAVES, GATED>(a, split, acc, smem, tid, wave, own);
}

}  // namespace
