// Gate, up, activation and product with bf16 weights: dlfp_gated_linear_bf16.
#include "dlfp_ffn.h"
#include "projection_choice.h"
#include "projection_gated.h"

namespace {

template <int BLOCKS, int TOKENS, int WAVES, int DEPTH>
int launch_few(const dlfp::ProjectionArgs& a, Grid g, dlfp::Split split, hipStream_t stream) {
  const int64_t tiles = g.down * g.across;
  gated_few_kernel<BLOCKS, TOKENS, WAVES, DEPTH>
      <<<(uint32_t)(tiles * split.splits), 64 * WAVES, 0, stream>>>(a, split);
  if (split.splits > 1) {
    constexpr int UNITS = BLOCKS / 2 * GatedFewShape<BLOCKS, TOKENS, WAVES, DEPTH>::TB;
    sum_few_kernel<BLOCKS, TOKENS, true><<<(uint32_t)(tiles * UNITS), 64, 0, stream>>>(
        a, (int)g.across, (int)tiles, split);
  }
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

template <int TN, int TM, int WAVES, int STAGES>
int launch_whole(const dlfp::ProjectionArgs& a, Grid g, dlfp::Split, hipStream_t stream) {
  split_kernel<TN, TM, WAVES, STAGES, true>
      <<<dim3((uint32_t)g.across, (uint32_t)g.down), 64 * WAVES, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

template <int TN, int TM, int WN, int WM, int STAGES>
int launch_tile(const dlfp::ProjectionArgs& a, Grid g, dlfp::Split split, hipStream_t stream) {
  const int64_t tiles = g.down * g.across;
  gated_tile_kernel<TN, TM, WN, WM, STAGES>
      <<<(uint32_t)(tiles * split.splits), 64 * WN * WM, 0, stream>>>(a, (int)g.down,
                                                                      (int)g.across, split);
  if (split.splits > 1)
    sum_tiles_kernel<TN, TM, WN, WM, true>
        <<<(uint32_t)(tiles * (TN * TM / 2048)), 256, 0, stream>>>(a, (int)g.down, (int)g.across,
                                                                   split);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

// Fitted to 500 sizes of 1-4096 tokens, 64-25600 features and columns, every variant with every
// split, weights read from memory.  The choice takes 1.031 times the fastest one's time on
// average (geometric mean; 1.08 in nine of ten sizes, 1.39 at worst).
#define FEW(B, T, W, D) 16 * B, T, 64 * W, W, BSTEP, 0, 0, true
#define WHOLE_K(TN, TM, W, STAGES) TN, TM, 64 * W, 0, 0, 0, 0, false
#define TILE(TN, TM, WN, WM, STAGES) TN, TM, 64 * WN * WM, 0, 0, 0, 0, true
#define FEW_CALLS(...) {nullptr, launch_few<__VA_ARGS__>}
#define WHOLE_K_CALLS(...) {nullptr, launch_whole<__VA_ARGS__>}
#define TILE_CALLS(...) {nullptr, launch_tile<__VA_ARGS__>}
constexpr Variant VARIANTS[] = {
    {FEW(2, 16, 4, 2), 0, {1.644f, 0.f, 0.f, 0.384f, 1.178f, 0.343f, 0.075f, 0.f, 0.f, 2.397f, 0.139f, 0.f}, FEW_CALLS(2, 16, 4, 2)},
    {FEW(2, 8, 4, 2), 0, {2.747f, 0.f, 0.f, 0.405f, 0.054f, 0.303f, 0.076f, 0.f, 0.f, 2.279f, 0.233f, 0.f}, FEW_CALLS(2, 8, 4, 2)},
    {FEW(2, 32, 4, 2), 0, {1.614f, 0.f, 0.f, 0.466f, 1.346f, 0.44f, 0.06f, 0.f, 0.f, 2.655f, 0.025f, 0.f}, FEW_CALLS(2, 32, 4, 2)},
    {WHOLE_K(64, 32, 4, 3), 0, {1.311f, 0.f, 0.f, 0.087f, 1.648f, 0.089f, 0.082f, 0.f, 0.f, 0.f, 0.f, 0.f}, WHOLE_K_CALLS(64, 32, 4, 3)},
    {WHOLE_K(32, 32, 8, 2), 0, {1.384f, 0.f, 0.f, 0.054f, 1.718f, 0.054f, 0.065f, 0.f, 0.f, 0.f, 0.f, 0.f}, WHOLE_K_CALLS(32, 32, 8, 2)},
    {TILE(128, 64, 4, 2, 3), 2, {1.978f, 0.f, 0.313f, 0.09f, 0.211f, 0.227f, 0.101f, 1.067f, 0.f, 2.497f, 0.092f, 0.f}, TILE_CALLS(128, 64, 4, 2, 3)},
    {TILE(256, 128, 4, 2, 3), 0, {1.077f, 0.f, 0.907f, 0.298f, 4.184f, 0.546f, 0.059f, 0.f, 0.f, 2.4f, 0.114f, 0.f}, TILE_CALLS(256, 128, 4, 2, 3)},
    {TILE(128, 32, 4, 1, 4), 2, {2.166f, 0.f, 0.058f, 0.033f, 0.354f, 0.171f, 0.122f, 0.78f, 0.f, 2.345f, 0.096f, 0.f}, TILE_CALLS(128, 32, 4, 1, 4)},
    {TILE(256, 256, 4, 2, 2), 0, {1.732f, 0.f, 2.072f, 0.544f, 5.764f, 1.041f, 0.04f, 0.f, 0.f, 0.396f, 0.109f, 0.f}, TILE_CALLS(256, 256, 4, 2, 2)},
    {TILE(128, 128, 2, 4, 4), 0, {1.279f, 0.f, 0.317f, 0.218f, 2.971f, 0.29f, 0.048f, 0.f, 0.f, 2.764f, 0.106f, 0.f}, TILE_CALLS(128, 128, 2, 4, 4)},
    {TILE(128, 64, 2, 2, 2), 3, {2.51f, 0.f, 0.424f, 0.126f, 0.061f, 0.052f, 0.102f, 0.524f, 0.349f, 2.655f, 0.126f, 0.f}, TILE_CALLS(128, 64, 2, 2, 2)},
};
#undef FEW
#undef WHOLE_K
#undef TILE
#undef FEW_CALLS
#undef WHOLE_K_CALLS
#undef TILE_CALLS

int launch(dlfp::ProjectionArgs& a, void* workspace, size_t bytes, hipStream_t stream) {
  (void)hipGetLastError();
  if (std::max<int64_t>(a.ldx, a.k) < dlfp::FAR_STRIDE)
    return launch_best(VARIANTS, true, a, (int64_t)a.n * a.k * 4, workspace, bytes, stream);
  const int64_t gm = ((int64_t)a.m + 63) / 64, gn = ((int64_t)a.n + 31) / 32;
  if (gm * gn * 256 > dlfp::MOST_THREADS) return DLFP_ERANGE;
  tile_kernel<64, 64, 2, 2, 4, true, true>
      <<<(uint32_t)(gm * gn), 256, 0, stream>>>(a, (int)gm, (int)gn);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

}  // namespace

namespace dlfp {

Form form_gated(int m, int n, int k, int64_t room) {
  return form_of(VARIANTS, true, m, n, k, (int64_t)n * k * 4, room);
}

}  // namespace dlfp

extern "C" int dlfp_gated_linear_bf16(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                                      const void* w_gate, const void* w_up, int32_t activation,
                                      void* out, int64_t ldo, int32_t out_dtype, void* workspace,
                                      size_t workspace_bytes, hipStream_t stream) {
  dlfp::ProjectionArgs a{static_cast<const uint16_t*>(x), {w_gate, w_up}, m, n, k, activation, ldx,
                         ldo, out, {nullptr, nullptr}, out_dtype, 0, 0};
  const int st = dlfp::check_projection(a, true, false, out_dtype, workspace);
  return st != DLFP_OK || m == 0 ? st : launch(a, workspace, workspace_bytes, stream);
}
