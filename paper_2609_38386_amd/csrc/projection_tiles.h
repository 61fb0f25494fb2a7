// Projections with bf16 weights in LDS tiles: out = x W^T (dlfp_linear_bf16) and, with
// GATED, act(x G^T) * (x U^T): of dlfp_gated_linear_bf16 the tiles of few features and
// tokens (split_kernel) and rows that are far apart (tile_kernel with FAR).
//
// The products are computed as out^T = W x^T on v_mfma_f32_32x32x16_bf16, so that a
// lane's accumulator holds four consecutive features of one token.  Two kernels share
// the operand layout:
//
//  - split_kernel (few output tiles): the wavefronts of a workgroup compute
//    the same tile over different 64-deep K steps, each from its own LDS ring
//    without a barrier, and add their results through LDS at the end;
//  - tile_kernel (many output tiles): the wavefronts own parts of the tile and
//    share LDS stages, one barrier per 64-deep K step.
//
// Stages are filled by direct global-to-LDS copies of whole 128-byte row
// segments: a copy instruction that covers 8 rows of 128 bytes moves 64 bytes
// per clock and CU, one of 16 rows of 64 bytes half of that (measured from L2,
// 34 against 17 TB/s over the chip), so the K step is 64 and never 32.
//
// A gated tile's 32-row blocks hold 16 rows of the gate and the 16 of the up
// projection that go with them: the accumulator rows 8 g + 4 (l / 32) + j of a lane
// are gates for g = 0, 1 and their ups for g = 2, 3, so that the activation and the
// product need no exchange, and everything before them is the plain product with
// twice the rows.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "projection.h"
#include "projection_device.h"

namespace {

constexpr int KSTEP = 64;              // k per LDS stage
constexpr int ROW_BYTES = KSTEP * 2;   // one 64-deep row of a stage
constexpr int COPY_ROWS = 8;           // rows of one copy instruction (64 lanes x 16 bytes)
constexpr int LDS_MAX = 160 * 1024;

typedef __attribute__((address_space(3))) char* lds_ptr_t;

__device__ __forceinline__ uint32_t lds_addr(char* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t)p);
}

// 16 bytes per lane from global memory straight into LDS at lds + 16 lane:
// base is wave-uniform, off the lane's byte offset.  The caller waits for the
// vector-memory counter before the data is read.
__device__ __forceinline__ void lds_copy16(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(lds)
               : "memory", "m0");
}
__device__ __forceinline__ void lds_copy16(const char* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(src), "s"(lds)
               : "memory", "m0");
}

// The same past the caches.
__device__ __forceinline__ void lds_stream16(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
               :
               : "v"(off), "s"(base), "s"(lds)
               : "memory", "m0");
}

// Wait until at most N of this wave's vector-memory operations are in flight.
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N <= 63, "the counter has six bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// The same, then meet the other waves; every LDS read of this wave has returned.
template <int N>
__device__ __forceinline__ void wait_copies_barrier() {
  static_assert(N <= 63, "the counter has six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Leave min(later, MOST) stages of L copies each in flight.
template <int MOST, int L, bool BARRIER>
__device__ __forceinline__ void wait_stages(int later) {
  if constexpr (MOST > 0) {
    if (later < MOST) return wait_stages<MOST - 1, L, BARRIER>(later);
  }
  if constexpr (BARRIER)
    wait_copies_barrier<MOST * L>();
  else
    wait_copies<MOST * L>();
}

// LDS layout of a stage: row r (64 k values, 128 bytes) keeps its 16-byte
// chunk c at position c ^ swz(r).  LDS serves sixteen lanes of a 16-byte read
// from 64 banks at once; two rows fill the banks, so the lanes that read the
// same chunk of sixteen rows are spread by bits 1-3 of the row (bits 0-2
// measured 1-4% slower: the even rows of a group then share positions).
__device__ __forceinline__ int swz(int row) { return (row >> 1) & 7; }

// Eight consecutive features of a token.  NEAR: the row stride of out fits 32 bits (a 64-bit product
// for every store took 1-2% of dlfp_linear_bf16's launches of short K: 545 tokens of 6144 x 1024
// 11.8 -> 12.0 us).
template <bool NEAR>
__device__ __forceinline__ void store8(const dlfp::ProjectionArgs& a, int m, int n, f32x4_t lo,
                                       f32x4_t hi) {
  const int64_t e = NEAR ? (int64_t)m * (int32_t)a.ldo + n : (int64_t)m * a.ldo + n;
  if (a.out_f32) {
    f32x4_t* o = reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + e);
    o[0] = lo;
    o[1] = hi;
    return;
  }
  uint16_t* o = static_cast<uint16_t*>(a.out) + e;
  const u32x4_t v = {pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]),
                     pack_bf16(hi[2], hi[3])};
  if (a.wide) {
    *reinterpret_cast<u32x4_t*>(o) = v;
  } else {
    reinterpret_cast<u32x2_t*>(o)[0] = u32x2_t{v[0], v[1]};
    reinterpret_cast<u32x2_t*>(o)[1] = u32x2_t{v[2], v[3]};
  }
}

// Per-lane byte offsets of the copies of ROWS rows by one wave: copy i covers
// rows first(i) .. + 8, lane l the 16-byte chunk that belongs at position
// l % 8 of row l / 8.  Rows past `last` re-read it (never stored).
template <int COUNT, typename F>
__device__ __forceinline__ void copy_offsets(uint32_t (&off)[COUNT], int lane, int ld, int last,
                                             F first) {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    const int r = first(i) + (lane >> 3);
    off[i] = (uint32_t)(min(r, last) * ld * 2 + (((lane & 7) ^ swz(r)) << 4));
  }
}

// Where the eight rows of copy c of a tile come from: which weights, and the first
// feature in the tile.  A gated tile alternates 16 rows of the gate and of the up.
template <bool GATED>
__device__ __forceinline__ constexpr int copy_weights(int c) {
  return GATED ? (c >> 1) & 1 : 0;
}
template <bool GATED>
__device__ __forceinline__ constexpr int copy_feature(int c) {
  return GATED ? 16 * (c >> 2) + 8 * (c & 1) : COPY_ROWS * c;
}

// The same for the rows of weights of copies copy(0), copy(1), ...
template <bool GATED, int COUNT, typename F>
__device__ __forceinline__ void weight_offsets(uint32_t (&off)[COUNT], int lane, int k, int last,
                                               F copy) {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    const int c = copy(i), f = copy_feature<GATED>(c) + (lane >> 3);
    off[i] = (uint32_t)(min(f, last) * k * 2 +
                        (((lane & 7) ^ swz(COPY_ROWS * c + (lane >> 3))) << 4));
  }
}

// The first row of tokens of a tile.  NEAR: row strides fit 32 bits.
template <bool NEAR>
__device__ __forceinline__ const char* token_rows(const dlfp::ProjectionArgs& a, int m0) {
  return reinterpret_cast<const char*>(a.x + (NEAR ? (int64_t)m0 * (int32_t)a.ldx : m0 * a.ldx));
}

// The first row of weights of a tile.
__device__ __forceinline__ const char* weight_rows(const dlfp::ProjectionArgs& a, int which,
                                                   int n0) {
  return static_cast<const char*>(a.weights[which]) + (int64_t)n0 * a.k * 2;
}

// The end of a tile whose K steps are split over the wavefronts: their sum, in wave order,
// for the first TOKENS tokens.  Every wave is done with LDS.  Plain ones are dlfp_linear_bf16's:
// whole tiles of features, row strides of 32 bits.
// A wave's accumulators are groups of four features: group (q, t, g) of lane l holds
// features 32 q + 8 g + 4 (l / 32) .. + 3 of token 32 t + l % 32.  A thread sums and stores
// eight consecutive features, neighbouring threads the next ones of the same token; the lane
// index is XORed with g and q so that both the writes and these reads spread over the banks.
template <int BN, int BM, int WAVES, int TOKENS, bool GATED>
__device__ __forceinline__ void store_sums(const dlfp::ProjectionArgs& a, f32x16_t (&acc)[BN][BM],
                                           char* smem, int tid, int wave, int n0, int m0) {
  constexpr int GROUPS = BN * BM * 256;
  const int lane = tid & 63;
  f32x4_t* res = reinterpret_cast<f32x4_t*>(smem);
  auto at = [](int q, int t, int g, int l) {
    return ((q * BM + t) * 4 + g) * 64 + (l ^ (g << 2) ^ ((q & 1) << 1));
  };
#pragma unroll
  for (int q = 0; q < BN; ++q)
#pragma unroll
    for (int t = 0; t < BM; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        res[wave * GROUPS + at(q, t, g, lane)] =
            f32x4_t{acc[q][t][4 * g], acc[q][t][4 * g + 1], acc[q][t][4 * g + 2],
                    acc[q][t][4 * g + 3]};
  __syncthreads();
  constexpr int EIGHTS = GATED ? 2 : 4;  // of features of a block
  for (int u = tid; u < EIGHTS * BN * TOKENS; u += 64 * WAVES) {
    const int g = u % EIGHTS, q = u / EIGHTS % BN, tok = u / EIGHTS / BN;
    auto sum = [&](int g, f32x4_t& lo, f32x4_t& hi) {
      const int ilo = at(q, tok >> 5, g, tok & 31), ihi = at(q, tok >> 5, g, 32 + (tok & 31));
      lo = res[ilo];
      hi = res[ihi];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) {
        lo += res[w * GROUPS + ilo];
        hi += res[w * GROUPS + ihi];
      }
    };
    f32x4_t lo, hi;
    sum(g, lo, hi);
    if constexpr (GATED) {
      f32x4_t ulo, uhi;
      sum(g + 2, ulo, uhi);
      lo = gated4(lo, ulo, a.act);
      hi = gated4(hi, uhi, a.act);
    }
    const int n = n0 + 8 * EIGHTS * q + 8 * g;
    if (m0 + tok < a.m && (!GATED || n < a.n)) store8<!GATED>(a, m0 + tok, n, lo, hi);
  }
}

// ---------------------------------------------------------------- split K

// One TN x TM tile per workgroup; wave w computes K steps w, w + WAVES, ...
// from its own ring of STAGES stages.  Few tiles leave most CUs one workgroup
// or none, and the launch is then bound by how fast a CU fills its LDS and by
// the memory latency in front of it: the ring keeps 64 KiB and more in flight
// per CU with no barrier to wait at, and every LDS byte is read once.
template <int TN, int TM, int WAVES, int STAGES, bool GATED = false>
__global__ __launch_bounds__(64 * WAVES) void split_kernel(dlfp::ProjectionArgs a) {
  constexpr int BN = TN / 32, BM = TM / 32;
  constexpr int NL = TN / COPY_ROWS, ML = TM / COPY_ROWS, L = NL + ML;
  constexpr int STAGE = (TN + TM) * ROW_BYTES;
  constexpr int RING = WAVES * STAGES * STAGE, RESULT = WAVES * TN * TM * 4;
  constexpr int LDS = RING > RESULT ? RING : RESULT;
  static_assert(LDS <= LDS_MAX, "LDS");
  __shared__ __attribute__((aligned(16))) char smem[LDS];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  constexpr int FEATURES = GATED ? TN / 2 : TN;
  const int n0 = blockIdx.x * FEATURES, m0 = blockIdx.y * TM;
  uint32_t woff[NL], xoff[ML];
  weight_offsets<GATED>(woff, lane, a.k, GATED ? a.n - 1 - n0 : TN - 1, [](int i) { return i; });
  copy_offsets(xoff, lane, a.ldx, a.m - 1 - m0, [](int i) { return COPY_ROWS * i; });
  const char* wbase[2] = {weight_rows(a, 0, n0), GATED ? weight_rows(a, 1, n0) : nullptr};
  const char* xbase = token_rows<!GATED>(a, m0);
  char* ring = smem + wave * (STAGES * STAGE);
  const uint32_t lds0 = lds_addr(ring);
  const int total = a.k / KSTEP;
  const int mine = total > wave ? (total - wave + WAVES - 1) / WAVES : 0;
  auto issue = [&](int i, int slot) {
    const int64_t ko = (int64_t)(wave + WAVES * i) * ROW_BYTES;
    const uint32_t d = lds0 + slot * STAGE;
#pragma unroll
    for (int j = 0; j < NL; ++j)
      lds_copy16(wbase[copy_weights<GATED>(j)] + ko, woff[j], d + j * 1024);
#pragma unroll
    for (int j = 0; j < ML; ++j) lds_copy16(xbase + ko, xoff[j], d + (NL + j) * 1024);
  };

  f32x16_t acc[BN][BM];
#pragma unroll
  for (int i = 0; i < BN; ++i)
#pragma unroll
    for (int j = 0; j < BM; ++j) acc[i][j] = f32x16_t{};
  // Operand reads: lane l takes row (l % 32) of a 32-row block and k
  // 8 (l / 32) .. + 8 of each 16-deep product.
  const int lr = lane & 31, lh = lane >> 5;
#pragma unroll
  for (int s = 0; s < STAGES; ++s)
    if (s < mine) issue(s, s);
  int slot = 0;
  for (int i = 0; i < mine; ++i) {
    wait_stages<STAGES - 1, L, false>(mine - 1 - i);
    const char* wl = ring + slot * STAGE + lr * ROW_BYTES;
    const char* xl = wl + TN * ROW_BYTES;
#pragma unroll
    for (int kk = 0; kk < KSTEP / 16; ++kk) {
      const int c = ((2 * kk + lh) ^ swz(lr)) << 4;
      bf16x8_t wf[BN], xf[BM];
#pragma unroll
      for (int q = 0; q < BN; ++q)
        wf[q] = *reinterpret_cast<const bf16x8_t*>(wl + 32 * q * ROW_BYTES + c);
#pragma unroll
      for (int q = 0; q < BM; ++q)
        xf[q] = *reinterpret_cast<const bf16x8_t*>(xl + 32 * q * ROW_BYTES + c);
#pragma unroll
      for (int q = 0; q < BN; ++q)
#pragma unroll
        for (int t = 0; t < BM; ++t)
          acc[q][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[q], xf[t], acc[q][t], 0, 0, 0);
    }
    wait_lds();  // the slot's reads have returned before it is refilled
    if (i + STAGES < mine) issue(i + STAGES, slot);
    slot = slot + 1 == STAGES ? 0 : slot + 1;
  }

  wait_copies_barrier<0>();  // every wave is done with its ring
  store_sums<BN, BM, WAVES, TM, GATED>(a, acc, smem, tid, wave, n0, m0);
}

// The end of a tile: through the wave's slice of LDS (`bytes` of them), so that whole
// runs of a row are stored (straight from the accumulators a store covers 16 bytes of 32
// rows; on m = 8192, n = 6144, k = 1024 the launch took 13% longer with those).  The
// wave's part of the tile starts at feature n0 and token m0; every wave is done with LDS.  WHOLE: all
// of its features are there, and row strides fit 32 bits (dlfp_linear_bf16).
template <int BN, int BM, int SLICE, bool GATED, bool WHOLE = false>
__device__ __forceinline__ void store_tile(const dlfp::ProjectionArgs& a, f32x16_t (&acc)[BN][BM],
                                           char* mine, int lane, int n0, int m0) {
  const int lr = lane & 31, lh = lane >> 5;
  constexpr int OF = GATED ? 16 : 32;      // features of a block
  constexpr int FB = GATED ? 4 : 2;        // blocks per pass
  static_assert(BN % FB == 0 || BN < FB, "passes");
  constexpr int B = BN < FB ? BN : FB;
  constexpr int RB = B * OF * 4 + 16;      // fp32 row of a pass, padded off the banks
  static_assert(SLICE >= 32 * RB, "epilogue slice");
#pragma unroll
  for (int j = 0; j < BM; ++j)
#pragma unroll
    for (int p = 0; p < BN / B; ++p) {
#pragma unroll
      for (int i = 0; i < B; ++i)
#pragma unroll
        for (int g = 0; g < OF / 8; ++g) {
          const f32x16_t& c = acc[p * B + i][j];
          f32x4_t v = {c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
          if constexpr (GATED)
            v = gated4(v, f32x4_t{c[8 + 4 * g], c[9 + 4 * g], c[10 + 4 * g], c[11 + 4 * g]}, a.act);
          *reinterpret_cast<f32x4_t*>(mine + lr * RB + (OF * i + 8 * g + 4 * lh) * 4) = v;
        }
      wait_lds();
      constexpr int PER_ROW = B * OF / 8, ROWS = 64 / PER_ROW;  // lanes per row, rows per store
#pragma unroll
      for (int r0 = 0; r0 < 32; r0 += ROWS) {
        const int r = r0 + lane / PER_ROW, f = 8 * (lane % PER_ROW);
        const f32x4_t* v = reinterpret_cast<const f32x4_t*>(mine + r * RB + f * 4);
        const int m = m0 + 32 * j + r, n = n0 + OF * p * B + f;
        if (m < a.m && (WHOLE || n < a.n)) store8<WHOLE>(a, m, n, v[0], v[1]);
      }
      wait_lds();
    }
}

// ---------------------------------------------------------------- tiles

// TN x TM tile per workgroup of WN x WM waves, STAGES shared LDS stages.  The
// operands of a 16-deep product are read from LDS while the one before it is
// on the matrix cores, across the stage barrier too.  FAR: 64-bit row offsets
// (row strides of 4 Mi elements and more).
template <int TN, int TM, int WN, int WM, int STAGES, bool FAR = false, bool GATED = false>
__global__ __launch_bounds__(64 * WN * WM, 2) void tile_kernel(dlfp::ProjectionArgs a, int gm, int gn) {
  constexpr int WAVES = WN * WM, BN = TN / WN / 32, BM = TM / WM / 32, KK = KSTEP / 16;
  constexpr int NL = TN / (COPY_ROWS * WAVES), ML = TM / (COPY_ROWS * WAVES), L = NL + ML;
  static_assert(NL * COPY_ROWS * WAVES == TN && ML * COPY_ROWS * WAVES == TM, "copies");
  constexpr int STAGE = (TN + TM) * ROW_BYTES;
  static_assert(STAGES * STAGE <= LDS_MAX, "LDS");
  __shared__ __attribute__((aligned(16))) char smem[STAGES * STAGE];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  // Workgroups are dealt round-robin over the 8 XCDs: each takes a contiguous
  // range of tiles, which walk the feature tiles in bands of 8 token tiles, so
  // the tiles running on an XCD share rows and weights in its L2.
  const int tiles = gm * gn, x = blockIdx.x & 7;
  const int t = x * (tiles >> 3) + min(x, tiles & 7) + (blockIdx.x >> 3);
  constexpr int BAND = 8;
  const int first = t / (BAND * gn) * BAND, h = min(BAND, gm - first), in = t - first * gn;
  constexpr int FEATURES = GATED ? TN / 2 : TN;
  const int n0 = (in / h) * FEATURES, m0 = (first + in % h) * TM;

  static_assert(!GATED || WAVES % 4 == 0, "the copies of a wave are of one weight");
  const char* wbase = weight_rows(a, copy_weights<GATED>(wave), n0);
  const int wlast = GATED ? a.n - 1 - n0 : TN - 1;
  const char* xbase = token_rows<!GATED>(a, m0);
  const int xlast = a.m - 1 - m0;
  uint32_t woff[NL], xoff[ML];
  if constexpr (!FAR) {
    weight_offsets<GATED>(woff, lane, a.k, wlast, [&](int i) { return i * WAVES + wave; });
    copy_offsets(xoff, lane, a.ldx, xlast, [&](int i) { return COPY_ROWS * (i * WAVES + wave); });
  }
  const uint32_t lds0 = lds_addr(smem) + wave * 1024;
  auto issue = [&](int ks, int slot) {
    const int64_t ko = (int64_t)ks * ROW_BYTES;
    const uint32_t d = lds0 + slot * STAGE;
    if constexpr (FAR) {
      auto src = [&](const char* base, int i, int first, int64_t ld, int last) {
        const int r = COPY_ROWS * (i * WAVES + wave) + (lane >> 3);
        return base + ko + min(first + (lane >> 3), last) * ld * 2 + (((lane & 7) ^ swz(r)) << 4);
      };
#pragma unroll
      for (int j = 0; j < NL; ++j)
        lds_copy16(src(wbase, j, copy_feature<GATED>(j * WAVES + wave), a.k, wlast),
                   d + j * WAVES * 1024);
#pragma unroll
      for (int j = 0; j < ML; ++j)
        lds_copy16(src(xbase, j, COPY_ROWS * (j * WAVES + wave), a.ldx, xlast),
                   d + TN * ROW_BYTES + j * WAVES * 1024);
    } else {
#pragma unroll
      for (int j = 0; j < NL; ++j) lds_copy16(wbase + ko, woff[j], d + j * WAVES * 1024);
#pragma unroll
      for (int j = 0; j < ML; ++j)
        lds_copy16(xbase + ko, xoff[j], d + TN * ROW_BYTES + j * WAVES * 1024);
    }
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

  const int steps = a.k / KSTEP;
#pragma unroll
  for (int s = 0; s < STAGES; ++s)
    if (s < steps) issue(s, s);
  wait_stages<STAGES - 1, L, true>(steps - 1);
  read(0, 0, 0);
  int slot = 0;
  for (int ks = 0; ks < steps; ++ks) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (kk + 1 < KK) {
        read(slot, kk + 1, (kk + 1) & 1);
      } else if (ks + 1 < steps) {
        // Stage ks + 1 has landed and no wave reads stage ks any more; its
        // slot takes stage ks + STAGES.
        const int next = slot + 1 == STAGES ? 0 : slot + 1;
        wait_stages<STAGES - 2, L, true>(steps - 2 - ks);
        read(next, 0, 0);
        if (ks + STAGES < steps) issue(ks + STAGES, slot);
        slot = next;
      }
      multiply(kk & 1);
    }
  }

  constexpr int SLICE = STAGES * STAGE / WAVES / 16 * 16;
  wait_copies_barrier<0>();
  store_tile<BN, BM, SLICE, GATED, !GATED>(a, acc, smem + wave * SLICE, lane,
                                           n0 + (GATED ? 16 : 32) * wn * BN, m0 + 32 * wm * BM);
}

}  // namespace
