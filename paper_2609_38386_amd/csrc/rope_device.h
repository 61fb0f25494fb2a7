// The position rotation of the append kernels.
//
// A row of 128 dims is held eight to a lane by 16 consecutive lanes (chunk c of
// a row in lane c).  The partner of a half pair, r / 2 dims away, is then r / 16
// lanes away (c ^ r / 16 inside the row), the partner of an interleaved pair in
// the lane itself, so a rotation takes no LDS of its own.  Angles come from a
// table in memory: a position's cosines and sines are 4 r bytes that every head
// of the token shares.
#ifndef DLFP_ROPE_DEVICE_H
#define DLFP_ROPE_DEVICE_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dlfp_cache.h"

namespace {

struct RopeArgs {
  const float* table;
  int positions;
  int rotary;       // 32, 64 or 128
  int interleaved;
};

// Cosines and sines of a chunk's eight dims (chunks past the rotary dims: some
// of the row's, not used).
struct Turn {
  float c[8], s[8];
};

__device__ __forceinline__ uint32_t rope_pack(float lo, float hi) {
  typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
  const pair_t v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

typedef float rope_f4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ Turn load_turn(const RopeArgs& r, int pos, int chunk) {
  Turn t;
  const int half = r.rotary >> 1;
  const float* row = r.table + (int64_t)pos * r.rotary;
  if (r.interleaved) {
    const float* at = row + ((4 * chunk) & (half - 1));
    const rope_f4_t c = *reinterpret_cast<const rope_f4_t*>(at);
    const rope_f4_t s = *reinterpret_cast<const rope_f4_t*>(at + half);
#pragma unroll
    for (int i = 0; i < 8; ++i) t.c[i] = c[i >> 1], t.s[i] = s[i >> 1];
    return t;
  }
  const float* at = row + ((8 * chunk) & (half - 1));
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const rope_f4_t c = *reinterpret_cast<const rope_f4_t*>(at + 4 * v);
    const rope_f4_t s = *reinterpret_cast<const rope_f4_t*>(at + half + 4 * v);
#pragma unroll
    for (int i = 0; i < 4; ++i) t.c[4 * v + i] = c[i], t.s[4 * v + i] = s[i];
  }
  return t;
}

// Products and sums rounded one by one, so that a key's code does not depend on
// how a kernel was compiled.
__device__ __forceinline__ float turned(float x, float partner, float c, float s, bool second) {
#pragma clang fp contract(off)
  const float a = x * c, b = partner * s;
  return second ? a + b : a - b;
}

// The rotated dims of chunk `chunk` (bf16 pairs x) in fp32.  Every lane of the
// row takes part.
__device__ __forceinline__ void rotate(const RopeArgs& r, const Turn& t, int chunk,
                                       const uint32_t x[4], float y[8]) {
  uint32_t other[4];
  const int away = r.rotary >> 4;
#pragma unroll
  for (int w = 0; w < 4; ++w) other[w] = __shfl_xor(x[w], away);
  const bool turns = 8 * chunk < r.rotary;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    auto half = [](uint32_t v, int odd) {
      return __builtin_bit_cast(float, odd ? v & 0xFFFF0000u : v << 16);
    };
    const float own = half(x[i >> 1], i & 1);
    const float partner = r.interleaved ? half(x[i >> 1], (i & 1) ^ 1) : half(other[i >> 1], i & 1);
    const bool second = r.interleaved ? i & 1 : 8 * chunk >= (r.rotary >> 1);
    y[i] = turns ? turned(own, partner, t.c[i], t.s[i], second) : own;
  }
}

struct QueryArgs {
  const uint16_t* q;
  uint16_t* out;
  int64_t ldq, ldo;
  int hq, chunks;  // query heads, groups of QUERY_HEADS of them
};

// Turns QUERY_HEADS heads of one token by one wavefront: four heads at a time, 16
// lanes a head, every load issued before the angles' (whose address waits for
// the position): an append of 2048 tokens, 16 and 8 heads, 11.5 us, 27.3 with
// eight tokens of a wavefront one after the other.  item: token * chunks + chunk of
// its heads.
constexpr int QUERY_HEADS = 16;
inline int query_chunks(int hq) { return (hq + QUERY_HEADS - 1) / QUERY_HEADS; }
__device__ __forceinline__ void rotate_queries(const QueryArgs& a, const RopeArgs& r,
                                               const int32_t* positions, int item) {
  const int lane = threadIdx.x & 63, chunk = lane & 15;
  const int t = item / a.chunks, h0 = item % a.chunks * QUERY_HEADS;
  const int n = min(QUERY_HEADS, a.hq - h0);
  const uint16_t* src = a.q + t * a.ldq + h0 * DLFP_HEAD_DIM + 8 * chunk;
  uint16_t* dst = a.out + t * a.ldo + h0 * DLFP_HEAD_DIM + 8 * chunk;
  const int pos = __builtin_amdgcn_readfirstlane(positions[t]);
  uint4 v[QUERY_HEADS / 4];
#pragma unroll
  for (int i = 0; i < QUERY_HEADS / 4; ++i)
    v[i] = *reinterpret_cast<const uint4*>(src + min(4 * i + (lane >> 4), n - 1) * DLFP_HEAD_DIM);
  if ((unsigned)pos >= (unsigned)r.positions) return;
  const Turn turn = load_turn(r, pos, chunk);
#pragma unroll
  for (int i = 0; i < QUERY_HEADS / 4; ++i) {
    const int head = 4 * i + (lane >> 4);
    const uint32_t x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
    float y[8];
    rotate(r, turn, chunk, x, y);
    const uint4 o = {rope_pack(y[0], y[1]), rope_pack(y[2], y[3]), rope_pack(y[4], y[5]),
                     rope_pack(y[6], y[7])};
    if (head < n) *reinterpret_cast<uint4*>(dst + head * DLFP_HEAD_DIM) = o;
  }
}

}  // namespace

#endif  // DLFP_ROPE_DEVICE_H
