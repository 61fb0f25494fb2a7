// Projections with 4-bit weights in LDS tiles, plain or gated: the tiles of
// projection_tiles.h with weights that stay codes until they are operands.
//
// A lane's 16 bytes of a row's codes are one group of 32 columns, the operands of four
// products; of a 64-deep K step it takes columns 32 (l / 32) .. + 32, so that a wave reads
// its codes from LDS once a step, an eighth of the bytes that bf16 operands would be, and
// widens eight codes in four instructions (exact, the group's exponent with them).
// Tokens come in 64-deep stages, weights in 256-deep ones, both as rows of 128 bytes, which
// is what the copies into LDS are fast with; a quarter of a weight stage is copied beside
// each token stage.
//
// The conversions (32 columns of a row block: 16 instructions) run beside the products at full
// rate, so that widening them once for the whole workgroup, through LDS, would only add traffic.
// Wavefronts are laid out along the features, since a wave widens its own rows and reads all
// tokens of its part: 256 x 256 tiles as 8 x 1 wavefronts run 4096 tokens of 12288 x 4096 in
// 314-318 us (1.30 PFLOP/s), as 4 x 2 in 347.  Large tiles are bound by what the power limit
// leaves of the matrix cores (57-65% busy), small ones by the latency of a step: its conditions,
// slots and waits took a third of it and are settled when the kernel is compiled (all stages but
// the last two; 4096 tokens of 12288 x 4096 360 -> 314 us).
//
// WHOLE: all operands of a step are read a step ahead, where the registers are there: tiles of
// 32 and 64 tokens (256 x 128 tiles lose by it, 2048 tokens of 4096 x 12288 169 -> 182 us).
#pragma once

#include <type_traits>

#include "projection_sums.h"

namespace {

constexpr int WSTEPS = 4;  // K steps of a weight stage

// The exponent bytes of eight groups of a row from group g on (fewer where the row ends), as
// the words that the lane's half reads: the byte of step s is byte 2 (s & 1) of word s >> 1.
__device__ __forceinline__ u32x2_t load_exps(const uint8_t* row, int g, int groups, int lh) {
  uint64_t v = 0;
  if (groups >= 8) {
    const int from = min(g, groups - 8);
    __builtin_memcpy(&v, row + from, 8);
    v >>= 8 * (g - from) + 8 * lh;
  } else {
    for (int i = 0; i < groups; i += 2) v |= (uint64_t)row[i + lh] << (8 * i);
  }
  return u32x2_t{(uint32_t)v, (uint32_t)(v >> 32)};
}

// The batch of copies of token stage t holds quarter (t + 3) % 4 of weight stage (t + 3) / 4,
// before the token rows, and goes out DEPTH steps ahead; a stage's slot is free again when
// the stage STAGES before it is done.
template <int TN, int TM, int WN, int WM, int DEPTH, int STAGES, bool GATED,
          bool WHOLE = false>
__global__ __launch_bounds__(64 * WN * WM, 2) void tile4_kernel(dlfp::ProjectionArgs a, int gm,
                                                                int gn, dlfp::Split split) {
  constexpr int WAVES = WN * WM, BN = TN / WN / 32, BM = TM / WM / 32, KK = KSTEP / 16;
  constexpr int ML = TM / (COPY_ROWS * WAVES);
  constexpr int QUARTER = TN / COPY_ROWS / WSTEPS;               // copies of a quarter stage
  constexpr int NL = QUARTER > WAVES ? QUARTER / WAVES : 1;      // of a wave, where it has any
  constexpr int TURNS = QUARTER < WAVES ? WAVES / QUARTER : 1;   // a wave has one in so many
  static_assert(ML * COPY_ROWS * WAVES == TM && QUARTER % 4 == 0 && WAVES % 4 == 0, "copies");
  static_assert(DEPTH >= 2 && DEPTH <= WSTEPS * STAGES - 6, "ring of weights");
  static_assert(WSTEPS % DEPTH == 0, "a step of a stage has its slot");
  // Copies of a wave behind the batch that a step waits for, at least: a step's own batch
  // goes out after it has waited, so that there are DEPTH - 2 of them.
  constexpr int BEHIND = (DEPTH - 2) * ML + (DEPTH - 2) / TURNS * NL;
  constexpr int XSTAGE = TM * ROW_BYTES, WSTAGE = TN * ROW_BYTES;
  constexpr int LDS = DEPTH * XSTAGE + STAGES * WSTAGE;
  static_assert(LDS <= LDS_MAX, "LDS");
  __shared__ __attribute__((aligned(16))) char smem[LDS];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  // Units (tiles of a split, split after split) of an XCD as tiles in tile_kernel.
  const int tiles = gm * gn, units = tiles * split.splits, xcd = blockIdx.x & 7;
  const int unit = xcd * (units >> 3) + min(xcd, units & 7) + (blockIdx.x >> 3);
  const int part = unit / tiles, t = unit - part * tiles;
  constexpr int BAND = 8;
  const int first = t / (BAND * gn) * BAND, h = min(BAND, gm - first), in = t - first * gn;
  constexpr int FEATURES = GATED ? TN / 2 : TN;
  const int n0 = (in / h) * FEATURES, m0 = (first + in % h) * TM;
  const int groups = a.k / 32, wlast = a.n - 1 - n0;
  const int all = (a.k / KSTEP + WSTEPS - 1) / WSTEPS;
  const int from = (int)((int64_t)all * part / split.splits);
  const int stages = (int)((int64_t)all * (part + 1) / split.splits) - from;
  const int steps = min(a.k / KSTEP - WSTEPS * from, WSTEPS * stages);

  // Copies: of tokens as in tile_kernel; of a quarter stage of weights copies
  // quarter * QUARTER + i WAVES + wave (with fewer than the waves, of some of them only).
  const char* xbase = reinterpret_cast<const char*>(a.x + (int64_t)m0 * a.ldx) +
                      (int64_t)from * (WSTEPS * ROW_BYTES);
  const int which = copy_weights<GATED>(wave);
  const char* wbase = static_cast<const char*>(a.weights[which]) + (int64_t)n0 * (a.k >> 1) +
                      (int64_t)from * ROW_BYTES;
  uint32_t xoff[ML], woff[WSTEPS][NL];
  copy_offsets(xoff, lane, (int)a.ldx, a.m - 1 - m0,
               [&](int i) { return COPY_ROWS * (i * WAVES + wave); });
  const int mine = QUARTER < WAVES ? wave % QUARTER : wave;
  const int chunk = lane & 7;
#pragma unroll
  for (int q = 0; q < WSTEPS; ++q)
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int c = q * QUARTER + i * WAVES + mine, r = COPY_ROWS * c + (lane >> 3);
      const int f = copy_feature<GATED>(c) + (lane >> 3);
      woff[q][i] = (uint32_t)(min(f, wlast) * (a.k >> 1) + ((chunk ^ swz(r)) << 4));
    }
  const uint32_t xlds = lds_addr(smem) + wave * 1024;
  const uint32_t wlds = lds_addr(smem) + DEPTH * XSTAGE + mine * 1024;
  // Quarter q of weight stage st.  Of a last stage that the row does not fill, copies past its
  // end take the stage's first group instead (never read).
  auto issue_w = [&](int st, int q, int slot) {
    if (QUARTER < WAVES && wave / QUARTER != q % TURNS) return;
    const char* src = wbase + (int64_t)st * ROW_BYTES;
    const int left = groups - 8 * (from + st);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      uint32_t off = woff[q][i];
      if (left < 8) {
        const int g = chunk ^ swz(COPY_ROWS * (q * QUARTER + i * WAVES + mine) + (lane >> 3));
        if (g >= left) off -= g << 4;
      }
      lds_copy16(src, off, wlds + slot * WSTAGE + (q * QUARTER + i * WAVES) * 1024);
    }
  };
  auto issue_x = [&](int t, int slot) {
    const char* src = xbase + (int64_t)t * ROW_BYTES;
#pragma unroll
    for (int j = 0; j < ML; ++j) lds_copy16(src, xoff[j], xlds + slot * XSTAGE + j * WAVES * 1024);
  };

  f32x16_t acc[BN][BM];
#pragma unroll
  for (int i = 0; i < BN; ++i)
#pragma unroll
    for (int j = 0; j < BM; ++j) acc[i][j] = f32x16_t{};
  const int lr = lane & 31, lh = lane >> 5, wn = wave / WM, wm = wave % WM;
  const char* xl = smem + (wm * BM * 32 + lr) * ROW_BYTES;
  const char* wl = smem + DEPTH * XSTAGE + (wn * BN * 32 + lr) * ROW_BYTES;
  // The lane's rows of exponents.
  const uint8_t* erow[BN];
#pragma unroll
  for (int q = 0; q < BN; ++q) {
    const int b = wn * BN + q;
    const int f = GATED ? 16 * b + (lr & 15) : 32 * b + lr;
    erow[q] = a.exps[GATED ? lr >> 4 : 0] + (int64_t)(n0 + min(f, wlast)) * groups;
  }
  u32x2_t exps[BN], later[BN];
  constexpr int SETS = WHOLE ? 2 : 1;
  u32x4_t codes[SETS][BN];
  bf16x8_t wf[2][BN], xf[WHOLE ? 2 * KK : 2][BM];
  auto read_x = [&](int slot, int kk, int set) {
    const int c = slot * XSTAGE + (((4 * lh + kk) ^ swz(lr)) << 4);
#pragma unroll
    for (int q = 0; q < BM; ++q)
      xf[set][q] = *reinterpret_cast<const bf16x8_t*>(xl + 32 * q * ROW_BYTES + c);
  };
  auto read_codes = [&](int slot, int s, int set = 0) {
    const int c = slot * WSTAGE + (((2 * s + lh) ^ swz(lr)) << 4);
#pragma unroll
    for (int q = 0; q < BN; ++q)
      codes[set][q] = *reinterpret_cast<const u32x4_t*>(wl + 32 * q * ROW_BYTES + c);
  };
  auto convert = [&](int s, int kk, int set, int from = 0) {
#pragma unroll
    for (int q = 0; q < BN; ++q) {
      const uint32_t word = s >> 1 ? exps[q][1] : exps[q][0];
      wf[set][q] = widen(codes[from][q][kk], scale_of((word >> (16 * (s & 1))) & 255u));
    }
  };
  auto multiply = [&](int wset, int xset) {
#pragma unroll
    for (int q = 0; q < BN; ++q)
#pragma unroll
      for (int u = 0; u < BM; ++u)
        acc[q][u] =
            __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[wset][q], xf[xset][u], acc[q][u], 0, 0, 0);
  };
  auto swap_exps = [&]() {
#pragma unroll
    for (int q = 0; q < BN; ++q) {
      exps[q] = later[q];
      asm volatile("" : "+v"(exps[q]));  // (here, where they have landed)
    }
  };
  auto next_exps = [&](int st) {
#pragma unroll
    for (int q = 0; q < BN; ++q) later[q] = load_exps(erow[q], 8 * (from + st), groups, lh);
  };
  // Step t's copies have landed, and every wave is done with the step before it.
  auto arrive = [&](auto inside, int t) {
    if (inside.value || ((t + DEPTH + 1) >> 2) < stages)
      wait_copies_barrier<BEHIND>();  // the batches behind are whole ones
    else
      wait_stages<DEPTH - 2, ML, true>(steps - 1 - t);
  };

#pragma unroll
  for (int q = 0; q < BN; ++q) exps[q] = load_exps(erow[q], 8 * from, groups, lh);
#pragma unroll
  for (int q = 0; q < BN; ++q)
    later[q] = load_exps(erow[q], 8 * (from + (stages > 1)), groups, lh);
#pragma unroll
  for (int q = 0; q < WSTEPS; ++q) issue_w(0, q, 0);
#pragma unroll
  for (int s = 0; s < DEPTH; ++s) {
    if (s && ((s + 3) >> 2) < stages) issue_w((s + 3) >> 2, (s + 3) & 3, ((s + 3) >> 2) % STAGES);
    if (s < steps) issue_x(s, s);
  }
  auto read_step = [&](int xslot, int wslot, int s, int set) {
    read_codes(wslot, s, set);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) read_x(xslot, kk, KK * set + kk);
  };
  arrive(std::false_type{}, 0);
  if constexpr (WHOLE) {
    read_step(0, 0, 0, 0);
  } else {
    read_x(0, 0, 0);
    read_codes(0, 0);
    convert(0, 0, 0);
  }
  // Step s of weight stage st.  `inside`: every step and stage that it looks ahead to is there,
  // so that no condition is left in it (they and the slots' arithmetic were a third of a step).
  int w0 = 0, w1 = 1 % STAGES, w2 = 2 % STAGES;  // slots of weight stages st to st + 2
  auto step = [&](auto inside, auto sc, int st) {
    constexpr int s = decltype(sc)::value, slot = s % DEPTH, next = (s + 1) % DEPTH;
    constexpr bool INSIDE = decltype(inside)::value, LAST = s + 1 == WSTEPS;
    const int ks = WSTEPS * st + s;
    // The next step: wait for it, read it as `read` does, and let the next copies go.
    auto advance = [&](auto read) {
      arrive(inside, ks + 1);
      if constexpr (LAST && !WHOLE) swap_exps();
      read(LAST ? w1 : w0);
      constexpr int ahead = (s + DEPTH + 3) >> 2;  // weight stage of batch ks + DEPTH
      static_assert(ahead == 1 || ahead == 2, "slots");
      if (INSIDE || st + ahead < stages)
        issue_w(st + ahead, (s + DEPTH + 3) & 3, ahead == 1 ? w1 : w2);
      if (INSIDE || ks + DEPTH < steps) issue_x(ks + DEPTH, slot);
      if constexpr (LAST && !WHOLE) {
        if (INSIDE || st + 2 < stages) next_exps(st + 2);
      }
    };
    if constexpr (WHOLE) {
      // All operands of the next step are read while this step's products run.
      if (INSIDE || ks + 1 < steps)
        advance([&](int w) { read_step(next, w, (s + 1) % WSTEPS, (s & 1) ^ 1); });
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        convert(s, kk, kk & 1, s & 1);
        multiply(kk & 1, KK * (s & 1) + kk);
      }
      if constexpr (LAST) {
        swap_exps();
        if (INSIDE || st + 2 < stages) next_exps(st + 2);
      }
    } else {
#pragma unroll
      for (int kk = 0; kk + 1 < KK; ++kk) {
        const int set = kk & 1;
        read_x(slot, kk + 1, set ^ 1);
        convert(s, kk + 1, set ^ 1);
        multiply(set, set);
        if constexpr (BN == 1 && BM == 4) {
          // A read of the next operands and half of a row block's conversions beside each product:
          // 2-3% of a 256 x 128 tile's time (2048 x 4096 x 12288 176 -> 172 us); other shapes lose
          // by it (256 x 256 9%).
#pragma unroll
          for (int i = 0; i < BN * BM; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
          }
        }
      }
      if (INSIDE || ks + 1 < steps)
        advance([&](int w) {
          read_x(next, 0, 0);
          read_codes(w, (s + 1) % WSTEPS);
        });
      multiply(1, 1);
      if (INSIDE || ks + 1 < steps) convert((s + 1) % WSTEPS, 0, 0);
    }
  };
  static_assert(KK % 2 == 0, "a step begins with set 0");
  auto stage = [&](auto inside, int st) {
    constexpr bool INSIDE = decltype(inside)::value;
    const int left = steps - WSTEPS * st;
    step(inside, std::integral_constant<int, 0>{}, st);
    if (INSIDE || left > 1) step(inside, std::integral_constant<int, 1>{}, st);
    if (INSIDE || left > 2) step(inside, std::integral_constant<int, 2>{}, st);
    if (INSIDE || left > 3) step(inside, std::integral_constant<int, 3>{}, st);
    const int first = w0;
    w0 = w1;
    w1 = STAGES == 2 ? first : w2;
    w2 = STAGES == 2 ? w0 : first;
  };
  // A stage looks ahead to two stages more, and to the steps of one.
  int st = 0;
  for (; st + 2 < stages; ++st) stage(std::true_type{}, st);
  for (; st < stages; ++st) stage(std::false_type{}, st);

  if (split.splits > 1) {
    store_parts(split, acc, (int64_t)unit * WAVES + wave, lane);
    return;
  }
  constexpr int SLICE = LDS / WAVES / 16 * 16;
  wait_copies_barrier<0>();
  store_tile<BN, BM, SLICE, GATED>(a, acc, smem + wave * SLICE, lane,
                                   n0 + (GATED ? 16 : 32) * wn * BN, m0 + 32 * wm * BM);
}

}  // namespace
