// Gate, up, activation and product with bf16 weights: dlfp_gated_linear_bf16.
#include "dlfp_ffn.h"
#include "projection_tiles.h"

namespace {

template <int TN, int TM, int WAVES, int STAGES>
int launch_split(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  const dim3 grid((a.n + TN / 2 - 1) / (TN / 2), (a.m + TM - 1) / TM);
  split_kernel<TN, TM, WAVES, STAGES, true><<<grid, 64 * WAVES, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}
template <int TN, int TM, int WN, int WM, int STAGES, bool FAR = false>
int launch_tile(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  const int64_t gm = ((int64_t)a.m + TM - 1) / TM, gn = ((int64_t)a.n + TN / 2 - 1) / (TN / 2);
  if (gm * gn * (64 * WN * WM) >= (int64_t)1 << 32) return DLFP_ERANGE;
  tile_kernel<TN, TM, WN, WM, STAGES, FAR, true>
      <<<(uint32_t)(gm * gn), 64 * WN * WM, 0, stream>>>(a, (int)gm, (int)gn);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

struct Variant {
  bool split;
  int tn, tm;
  float start, step, round, work;
  int (*launch)(const dlfp::ProjectionArgs&, hipStream_t);
};
constexpr Variant VARIANTS[] = {
    {true, 32, 32, 1.35f, -0.024f, 0.80f, 0.120f, launch_split<32, 32, 8, 2>},
    {true, 64, 32, 1.30f, -0.029f, 1.05f, 0.170f, launch_split<64, 32, 4, 3>},
    {true, 64, 64, 1.44f, -0.043f, 1.64f, 0.231f, launch_split<64, 64, 4, 2>},
    {false, 128, 64, 1.79f, 0.065f, 0.91f, 0.305f, launch_tile<128, 64, 2, 2, 3>},
    {false, 128, 128, 1.05f, -0.060f, 2.41f, 0.545f, launch_tile<128, 128, 2, 4, 4>},
    {false, 128, 256, 0.54f, -0.142f, 3.93f, 0.942f, launch_tile<128, 256, 2, 4, 3>},
    {false, 256, 256, -0.42f, -0.277f, 6.99f, 1.657f, launch_tile<256, 256, 2, 4, 2>},
};
constexpr int CUS = 256;
constexpr int MOST_GRID_Y = 65535;
// Row strides from here on take 64-bit offsets (255 rows of 2 bytes each fit
// 32 bits below).
constexpr int FAR_STRIDE = 1 << 22;

int launch(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  (void)hipGetLastError();
  if (std::max<int64_t>(a.ldx, a.k) >= FAR_STRIDE)
    return launch_tile<64, 64, 2, 2, 4, true>(a, stream);
  const Variant* best = nullptr;
  float least = 0.f;
  for (const Variant& v : VARIANTS) {
    const int64_t down = ((int64_t)a.m + v.tm - 1) / v.tm;
    if (v.split && down > MOST_GRID_Y) continue;
    const int64_t tiles = down * ((2 * (int64_t)a.n + v.tn - 1) / v.tn);
    const float rounds = (float)((tiles + CUS - 1) / CUS), steps = (float)(a.k / KSTEP);
    const float t = v.start + v.step * steps + (v.round + v.work * steps) * rounds;
    if (!best || t < least) {
      best = &v;
      least = t;
    }
  }
  return best->launch(a, stream);
}

}  // namespace

extern "C" int dlfp_gated_linear_bf16(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                                      const void* w_gate, const void* w_up, int32_t activation,
                                      void* out, int64_t ldo, int32_t out_dtype, void* workspace,
                                      size_t workspace_bytes, hipStream_t stream) {
  dlfp::ProjectionArgs a{static_cast<const uint16_t*>(x), {w_gate, w_up}, {nullptr, nullptr}, out,
                         ldx, ldo, m, n, k, activation, out_dtype, 0};
  const int st = dlfp::check_projection(a, true, false, out_dtype, workspace);
  return st != DLFP_OK || m == 0 ? st : launch(a, stream);
}
