// Gate, up, activation and product with bf16 weights: dlfp_gated_linear_bf16.
#include "dlfp_ffn.h"
#include "projection_vector.h"

extern "C" int dlfp_gated_linear_bf16(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                                      const void* w_gate, const void* w_up, int32_t activation,
                                      void* out, int64_t ldo, int32_t out_dtype,
                                      hipStream_t stream) {
  const dlfp::ProjectionArgs a{static_cast<const uint16_t*>(x), {w_gate, w_up}, {nullptr, nullptr},
                               out, ldx, ldo, m, n, k, activation, out_dtype, 0};
  const int st = dlfp::check_projection(a, true, false, out_dtype);
  return st != DLFP_OK || m == 0 ? st : launch_vector<false, true, 1, 8>(a, stream);
}
