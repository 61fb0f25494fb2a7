// What the projection entry points of dlfp_ffn.h share: arguments, their checks and launches.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace dlfp {

// out = x W^T, or act(x G^T) * (x U^T): weights [0] are W or G, [1] are U.
// What a kernel needs before its first copies comes first, in one line of 64 bytes.
struct ProjectionArgs {
  const uint16_t* x;
  const void* weights[2];        // bf16, or codes
  int32_t m, n, k, act;
  int64_t ldx, ldo;
  void* out;
  const uint8_t* exps[2];        // of codes
  int32_t out_f32;
  int32_t wide;    // bf16 output rows take 16-byte stores
  int32_t stream;  // weights are read past the caches
};

// A launch whose K is split over `splits` workgroups a tile: the partial sums go to `part`,
// [split][tile][unit of four features of a token] fp32, and a second launch adds them.
struct Split {
  float* part;
  int32_t splits;
};

// Row strides from here on take 64-bit offsets (255 rows of 2 bytes each fit 32 bits below).
constexpr int FAR_STRIDE = 1 << 22;

// Tokens and features at most, so that the index of a tile's last row fits 31 bits.
constexpr int MOST_ROWS = 0x7fffffff - 1024;

// Threads of a launch at most.
constexpr int64_t MOST_THREADS = ((int64_t)1 << 32) - 1;

// Outputs from here on are more threads than that in any form (512 for each 256 x 256 at least),
// below it the products of sizes that the choice takes fit 63 bits.
constexpr int64_t MOST_OUTPUTS = (int64_t)1 << 39;
inline bool too_many(int m, int n) {
  return m > MOST_ROWS || n > MOST_ROWS || (int64_t)m * n >= MOST_OUTPUTS;
}

// Few tokens with 4-bit weights: bytes between the exponents of rows in LDS.  All of K: as in
// memory; a split of it: its own groups, and up to 15 before them that a 16-byte piece begins with.
inline __host__ __device__ int exps_pitch(int k, int splits, int step_columns) {
  if (splits == 1) return k / 32;
  const int steps = (k + step_columns - 1) / step_columns;
  return ((steps + splits - 1) / splits * (step_columns / 32) + 30) / 16 * 16;
}
// Bytes of 16 rows of them, in whole copies.
inline __host__ __device__ int exps_bytes(int k, int splits, int step_columns) {
  return (16 * exps_pitch(k, splits, step_columns) + 1023) / 1024 * 1024;
}

// The form that a call of near rows takes with `room` bytes of workspace: its place among the
// variants (-1: a launch of none can have the threads), its tile, its splits and their bytes, and
// whether weights are read past the caches.
struct Form {
  int variant, rows, tokens, splits, stream;
  int64_t bytes;
};
Form form_w4(bool gated, int m, int n, int k, int64_t room);
Form form_gated(int m, int n, int k, int64_t room);

constexpr int64_t MOST_PARTS = 32 << 20;  // bytes of partial sums

// DLFP_OK, or what is wrong with them; sets wide.
int check_projection(ProjectionArgs& a, bool gated, bool codes, int32_t out_dtype,
                     const void* workspace);

}  // namespace dlfp
