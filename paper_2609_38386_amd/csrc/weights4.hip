// Weights to 4 bits and back (the format of dlfp_ffn.h).
//
// A thread holds 8 columns and four neighbours a group of 32: the group's largest
// magnitude is a maximum over their bit patterns, exchanged between the four lanes with
// no shared memory, and its exponent follows from that pattern's fields, with no
// logarithm; codes are the conversion instruction's.  16 bytes are read or written a lane,
// whole rows by neighbouring lanes.  Bound by the bytes (2 + 17/32 a weight): 25600 x 5120
// takes 71 us to 4 bits and 53 us back (4.7 and 6.4 TB/s; a large copy reaches 5.1), 1024 x
// 2048 2.6 us, of which 2 are the launch.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "dlfp_ffn.h"
#include "projection_device.h"

namespace {

constexpr int THREADS = 256;

// (by value: a bit cast of a vector's element itself reads the vector's first)
__device__ __forceinline__ bf16x2_t pair(uint32_t bits) {
  return __builtin_bit_cast(bf16x2_t, bits);
}

__global__ __launch_bounds__(THREADS) void quantize_kernel(const uint16_t* w, int64_t ldw,
                                                           uint32_t* codes, uint8_t* exps,
                                                           int32_t per_row, uint32_t total) {
  const uint32_t i = blockIdx.x * THREADS + threadIdx.x;
  if (i >= total) return;  // (whole groups of four threads: per_row is a multiple of 4)
  const uint32_t row = i / (uint32_t)per_row, c = i - row * (uint32_t)per_row;
  const u32x4_t v = *reinterpret_cast<const u32x4_t*>(w + (int64_t)row * ldw + 8 * c);
  // Bit patterns without the sign grow with the magnitude, past all others where a
  // value is infinite or NaN.
  uint32_t most = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    most = max(most, max(v[j] & 0x7fffu, (v[j] >> 16) & 0x7fffu));
  most = max(most, (uint32_t)__shfl_xor((int)most, 1));
  most = max(most, (uint32_t)__shfl_xor((int)most, 2));
  // 1.f 2^E <= 6 2^e = 1.5 2^(e + 2): e = E - 2 up to a fraction of one half, else E - 1.
  const int power = (int)(most >> 7) + ((most & 127u) > 64u ? -1 : -2);
  const bool finite = most < 0x7f80u;
  const uint32_t byte = finite ? (uint32_t)min(max(power, 2), 252) : 255u;
  const float scale = scale_of(byte);
  uint32_t out = 0;
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, pair(v[0]), scale, 0);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, pair(v[1]), scale, 1);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, pair(v[2]), scale, 2);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, pair(v[3]), scale, 3);
  codes[i] = finite ? out : 0u;
  if ((i & 3) == 0) exps[i >> 2] = (uint8_t)byte;
}

__global__ __launch_bounds__(THREADS) void dequantize_kernel(const uint32_t* codes,
                                                             const uint8_t* exps, uint16_t* w,
                                                             int64_t ldw, int32_t per_row,
                                                             uint32_t total) {
  const uint32_t i = blockIdx.x * THREADS + threadIdx.x;
  if (i >= total) return;
  const uint32_t row = i / (uint32_t)per_row, c = i - row * (uint32_t)per_row;
  *reinterpret_cast<bf16x8_t*>(w + (int64_t)row * ldw + 8 * c) =
      widen(codes[i], scale_of(exps[i >> 2]));
}

int check(int32_t n, int32_t k, const void* w, int64_t ldw, const void* codes, const void* exps) {
  if (n < 0 || k <= 0) return DLFP_EINVAL;
  if (k % DLFP_W4_GROUP) return DLFP_EUNSUPPORTED;
  if (ldw < k || ldw % 8) return DLFP_EINVAL;
  if (n == 0) return DLFP_OK;
  if (!w || !codes || !exps) return DLFP_EINVAL;
  if ((reinterpret_cast<uintptr_t>(w) | reinterpret_cast<uintptr_t>(codes)) & 15)
    return DLFP_EINVAL;
  if ((int64_t)n * k >= (int64_t)1 << 34) return DLFP_ERANGE;
  return DLFP_OK;
}

}  // namespace

extern "C" int dlfp_quantize_w4(int32_t n, int32_t k, const void* w, int64_t ldw, void* codes,
                                void* exps, hipStream_t stream) {
  const int st = check(n, k, w, ldw, codes, exps);
  if (st != DLFP_OK || n == 0) return st;
  const uint32_t total = (uint32_t)((int64_t)n * k / 8);
  (void)hipGetLastError();
  quantize_kernel<<<(total + THREADS - 1) / THREADS, THREADS, 0, stream>>>(
      static_cast<const uint16_t*>(w), ldw, static_cast<uint32_t*>(codes),
      static_cast<uint8_t*>(exps), k / 8, total);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

extern "C" int dlfp_dequantize_w4(int32_t n, int32_t k, const void* codes, const void* exps,
                                  void* w, int64_t ldw, hipStream_t stream) {
  const int st = check(n, k, w, ldw, codes, exps);
  if (st != DLFP_OK || n == 0) return st;
  const uint32_t total = (uint32_t)((int64_t)n * k / 8);
  (void)hipGetLastError();
  dequantize_kernel<<<(total + THREADS - 1) / THREADS, THREADS, 0, stream>>>(
      static_cast<const uint32_t*>(codes), static_cast<const uint8_t*>(exps),
      static_cast<uint16_t*>(w), ldw, k / 8, total);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}
