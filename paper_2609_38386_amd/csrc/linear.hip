// Dense projections of one transformer layer's tokens, for the full-iteration
// latency of Eq. 1: the iteration cost the controller observes includes the
// linear layers, whose work grows with the prefill chunk p_t (Sec. 2.1), not
// only the attention.
//
//   out[m][n] = sum_k x[m][k] w[n][k]      (bf16 in, fp32 accumulation)
//
// x is row-major with row stride ldx (elements), w is [n][k] (a linear layer's
// weight as stored: one row per output feature), out row-major with row stride
// ldo.  The kernels are those of projection_tiles.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "dlfp.h"
#include "projection_tiles.h"

namespace {

constexpr int N_UNIT = 128;            // n is a multiple of this

template <int TN, int TM, int WAVES, int STAGES>
void launch_split(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  const dim3 grid(a.n / TN, (a.m + TM - 1) / TM);
  split_kernel<TN, TM, WAVES, STAGES><<<grid, 64 * WAVES, 0, stream>>>(a);
}
template <int TN, int TM, int WN, int WM, int STAGES, bool FAR = false>
void launch_tile(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  const int gm = (a.m + TM - 1) / TM, gn = a.n / TN;
  tile_kernel<TN, TM, WN, WM, STAGES, FAR><<<gm * gn, 64 * WN * WM, 0, stream>>>(a, gm, gn);
}

// Which kernel and tile: the one whose estimated time is lowest.  With
// r = ceil(tiles / 256) rounds over the CUs and s = k / 64 K steps the estimate
// is start + step s + (round + work s) r microseconds, fitted to 660 launches of
// 1-8192 tokens times 24 (n, k), the Qwen3-0.6B, 8B and 32B projections among them
// (relative errors; sizes where a variant takes over 1.8 times the best one's
// time count little).  There the choice is within 0.4% of the fastest variant on
// average, and against one 128 x 128 tile for every size, as before, the launches
// take 0.42x of the time (geometric mean) and none takes longer: n = k = 1024
// 11.0 -> 3.3 us at m = 32, 14.3 -> 6.3 us at m = 545, 28.2 -> 21.3 us at
// m = 8192; n = 6144, k = 1024, m = 8192 141.5 -> 104.5 us; n = 1024, k = 3072,
// m = 545 36.9 -> 12.1 us; n = 5120, k = 8192, m = 4096 384 -> 353 us.  (A row's
// sum over k runs in another order in another kernel, so its last bit can depend
// on the number of rows.)  Small tiles win where the tiles are few, since
// every CU then fills its LDS side by side; large ones where the tiles fill
// the chip, since each operand byte then serves more products.
struct Variant {
  int tn, tm;
  float start, step, round, work;
  void (*launch)(const dlfp::ProjectionArgs&, hipStream_t);
};
constexpr Variant VARIANTS[] = {
    {32, 32, 1.35f, -0.024f, 0.80f, 0.120f, launch_split<32, 32, 8, 2>},
    {64, 32, 1.30f, -0.029f, 1.05f, 0.170f, launch_split<64, 32, 4, 3>},
    {64, 64, 1.44f, -0.043f, 1.64f, 0.231f, launch_split<64, 64, 4, 2>},
    {128, 64, 1.79f, 0.065f, 0.91f, 0.305f, launch_tile<128, 64, 2, 2, 3>},
    {128, 128, 1.05f, -0.060f, 2.41f, 0.545f, launch_tile<128, 128, 2, 4, 4>},
    {128, 256, 0.54f, -0.142f, 3.93f, 0.942f, launch_tile<128, 256, 2, 4, 3>},
    {256, 256, -0.42f, -0.277f, 6.99f, 1.657f, launch_tile<256, 256, 2, 4, 2>},
};
constexpr int CUS = 256;
// Row strides from here on take 64-bit offsets (255 rows of 2 bytes each fit
// 32 bits below).
constexpr int FAR_STRIDE = 1 << 22;

void launch_linear(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  if (std::max<int64_t>(a.ldx, a.k) >= FAR_STRIDE) return launch_tile<64, 64, 2, 2, 4, true>(a, stream);
  const Variant* best = nullptr;
  float least = 0.f;
  for (const Variant& v : VARIANTS) {
    if (a.n % v.tn) continue;
    const int64_t tiles = ((int64_t)a.m + v.tm - 1) / v.tm * (a.n / v.tn);
    const float rounds = (float)((tiles + CUS - 1) / CUS), steps = (float)(a.k / KSTEP);
    const float t = v.start + v.step * steps + (v.round + v.work * steps) * rounds;
    if (!best || t < least) {
      best = &v;
      least = t;
    }
  }
  best->launch(a, stream);
}

}  // namespace

extern "C" int dlfp_linear_bf16(int32_t m, int32_t n, int32_t k, const void* x, int32_t ldx,
                                const void* w, void* out, int32_t ldo, int32_t out_dtype,
                                hipStream_t stream) {
  if (m < 0 || n <= 0 || k <= 0) return DLFP_EINVAL;
  if (out_dtype != 0 && out_dtype != 1) return DLFP_EINVAL;
  if (n % N_UNIT || k % KSTEP) return DLFP_EUNSUPPORTED;
  if (ldx < k || ldo < n || ldx % 8 || ldo % 4) return DLFP_EINVAL;
  if (m == 0) return DLFP_OK;
  if (!x || !w || !out) return DLFP_EINVAL;
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(w)) & 15) return DLFP_EINVAL;
  if (reinterpret_cast<uintptr_t>(out) & (out_dtype ? 15 : 7)) return DLFP_EINVAL;
  const bool wide = (reinterpret_cast<uintptr_t>(out) & 15) == 0 && ldo % 8 == 0;
  const dlfp::ProjectionArgs a{static_cast<const uint16_t*>(x), {w, nullptr}, m, n, k, 0, ldx, ldo,
                               out, {nullptr, nullptr}, out_dtype, wide, 0};
  (void)hipGetLastError();
  launch_linear(a, stream);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}
