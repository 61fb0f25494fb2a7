// Projections with 4-bit weights: dlfp_linear_w4, dlfp_gated_linear_w4.
#include "dlfp_ffn.h"
#include "projection_vector.h"

namespace dlfp {

int check_projection(ProjectionArgs& a, bool gated, bool codes, int32_t out_dtype) {
  if (a.m < 0 || a.n <= 0 || a.k <= 0) return DLFP_EINVAL;
  if (out_dtype != 0 && out_dtype != 1) return DLFP_EINVAL;
  if (gated && a.act != DLFP_SILU && a.act != DLFP_GELU) return DLFP_EINVAL;
  if (a.n % 16 || a.k % 64) return DLFP_EUNSUPPORTED;
  if (a.ldx < a.k || a.ldo < a.n || a.ldx % 8 || a.ldo % 4) return DLFP_EINVAL;
  if (a.m == 0) return DLFP_OK;
  if (!a.x || !a.out || (reinterpret_cast<uintptr_t>(a.x) & 15)) return DLFP_EINVAL;
  if (reinterpret_cast<uintptr_t>(a.out) & (out_dtype ? 15 : 7)) return DLFP_EINVAL;
  for (int i = 0; i < (gated ? 2 : 1); ++i) {
    if (!a.weights[i] || (reinterpret_cast<uintptr_t>(a.weights[i]) & 15)) return DLFP_EINVAL;
    if (codes && !a.exps[i]) return DLFP_EINVAL;
  }
  a.wide = (reinterpret_cast<uintptr_t>(a.out) & 15) == 0 && a.ldo % 8 == 0;
  return DLFP_OK;
}

}  // namespace dlfp

namespace {

template <bool GATED>
int launch(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  return launch_vector<true, GATED, 1, 8>(a, stream);
}

}  // namespace

extern "C" int dlfp_linear_w4(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                              const void* codes, const void* exps, void* out, int64_t ldo,
                              int32_t out_dtype, hipStream_t stream) {
  dlfp::ProjectionArgs a{static_cast<const uint16_t*>(x),
                               {codes, nullptr},
                               {static_cast<const uint8_t*>(exps), nullptr},
                               out, ldx, ldo, m, n, k, 0, out_dtype, 0};
  const int st = dlfp::check_projection(a, false, true, out_dtype);
  return st != DLFP_OK || m == 0 ? st : launch<false>(a, stream);
}

extern "C" int dlfp_gated_linear_w4(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                                    const void* gate_codes, const void* gate_exps,
                                    const void* up_codes, const void* up_exps, int32_t activation,
                                    void* out, int64_t ldo, int32_t out_dtype,
                                    hipStream_t stream) {
  dlfp::ProjectionArgs a{
      static_cast<const uint16_t*>(x),
      {gate_codes, up_codes},
      {static_cast<const uint8_t*>(gate_exps), static_cast<const uint8_t*>(up_exps)},
      out, ldx, ldo, m, n, k, activation, out_dtype, 0};
  const int st = dlfp::check_projection(a, true, true, out_dtype);
  return st != DLFP_OK || m == 0 ? st : launch<true>(a, stream);
}
