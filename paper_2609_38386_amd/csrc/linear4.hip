// Projections with 4-bit weights: dlfp_linear_w4, dlfp_gated_linear_w4.  The kernels are those
// of projection_few4.h and projection_tiles4.h, and a plain one for rows that are far apart.
#include "dlfp_ffn.h"
#include "projection_choice.h"
#include "projection_few4.h"
#include "projection_tiles4.h"

namespace {

using dlfp::FAR_STRIDE;

// ---------------------------------------------------------------- far rows

// Rows of x or of weights 2^22 elements and more apart: 16 features and 16 tokens a workgroup,
// operands straight from memory with 64-bit addresses, K over eight wavefronts in steps of 128
// columns.  (The other kernels' copies have 32-bit offsets from a tile's first row.)  Simple, since
// no program lays tokens out so: bound by the address unit, and weights are read again for every
// 16 tokens (64 tokens of 4096 x 4096, timed with a call's events: 24 us, 14 where rows are
// near; 256 tokens: 70 and 27).
constexpr int FAR_WAVES = 8, FAR_STEP = 128;

template <bool GATED>
__global__ __launch_bounds__(64 * FAR_WAVES) void far4_kernel(dlfp::ProjectionArgs a) {
  constexpr int B = GATED ? 2 : 1;
  __shared__ f32x4_t sums[FAR_WAVES][B][64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, lr = lane & 15, quad = lane >> 4;
  const uint32_t gn = (uint32_t)a.n / 16;
  const int n0 = (int)(blockIdx.x % gn) * 16, m0 = (int)(blockIdx.x / gn) * 16;
  const uint16_t* x = a.x + (int64_t)min(m0 + lr, a.m - 1) * a.ldx;
  f32x4_t acc[B] = {};
  // (k0 itself passes 31 bits behind the last step of the longest rows)
  for (uint32_t k0 = FAR_STEP * wave; k0 < (uint32_t)a.k; k0 += FAR_STEP * FAR_WAVES) {
    // Of a last step of 64 columns half of the lanes' columns are past the row: zeros.
    const int c = (int)k0 + 32 * quad;
    const bool in = c < a.k;
    bf16x8_t xf[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
      xf[t] = in ? *reinterpret_cast<const bf16x8_t*>(x + c + 8 * t) : bf16x8_t{};
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int64_t row = n0 + lr;
      const char* codes = static_cast<const char*>(a.weights[b]) + row * (a.k >> 1);
      const u32x4_t w = in ? *reinterpret_cast<const u32x4_t*>(codes + (c >> 1)) : u32x4_t{};
      const float scale = scale_of(in ? a.exps[b][row * (a.k >> 5) + (c >> 5)] : 0);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        acc[b] =
            __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w[t], scale), xf[t], acc[b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int b = 0; b < B; ++b) sums[wave][b][lane] = acc[b];
  __syncthreads();
  if (wave) return;
  f32x4_t v = sums[0][0][lane], up = sums[0][B - 1][lane];
#pragma unroll
  for (int w = 1; w < FAR_WAVES; ++w) {
    v += sums[w][0][lane];
    up += sums[w][B - 1][lane];
  }
  if constexpr (GATED) v = gated4(v, up, a.act);
  if (m0 + lr < a.m) store4(a, m0 + lr, n0 + 4 * quad, v);
}

template <bool GATED>
int launch_far(const dlfp::ProjectionArgs& a, hipStream_t stream) {
  const int64_t blocks = (int64_t)(a.n / 16) * (((int64_t)a.m + 15) / 16);
  if (blocks * (64 * FAR_WAVES) > dlfp::MOST_THREADS) return DLFP_ERANGE;
  far4_kernel<GATED><<<(uint32_t)blocks, 64 * FAR_WAVES, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

// ---------------------------------------------------------------- launches

template <bool GATED, int BLOCKS, int TOKENS, int WAVES, int DEPTH, int HALVES>
int launch_few(const dlfp::ProjectionArgs& a, Grid g, dlfp::Split split, hipStream_t stream) {
  using Shape = FewShape<BLOCKS, TOKENS, WAVES, DEPTH, HALVES>;
  const int64_t tiles = g.down * g.across;
  few4_kernel<BLOCKS, TOKENS, WAVES, DEPTH, HALVES, GATED>
      <<<(uint32_t)(tiles * split.splits), 64 * WAVES, (size_t)Shape::lds(a.k, split.splits),
         stream>>>(a, split);
  if (split.splits > 1) {
    constexpr int UNITS = (GATED ? BLOCKS / 2 : BLOCKS) * Shape::TB;
    sum_few_kernel<BLOCKS, TOKENS, GATED><<<(uint32_t)(tiles * UNITS), 64, 0, stream>>>(
        a, (int)g.across, (int)tiles, split);
  }
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

template <bool GATED, int TN, int TM, int WN, int WM, int DEPTH, int STAGES, bool WHOLE>
int launch_tile(const dlfp::ProjectionArgs& a, Grid g, dlfp::Split split, hipStream_t stream) {
  const int64_t tiles = g.down * g.across;
  tile4_kernel<TN, TM, WN, WM, DEPTH, STAGES, GATED, WHOLE>
      <<<(uint32_t)(tiles * split.splits), 64 * WN * WM, 0, stream>>>(a, (int)g.down,
                                                                      (int)g.across, split);
  if (split.splits > 1) {
    constexpr int BLOCKS = TN * TM / 16 * (GATED ? 2 : 4) / 256;
    sum_tiles_kernel<TN, TM, WN, WM, GATED><<<(uint32_t)(tiles * BLOCKS), 256, 0, stream>>>(
        a, (int)g.down, (int)g.across, split);
  }
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

// ---------------------------------------------------------------- choice

template <int BLOCKS, int TOKENS, int WAVES, int DEPTH, int HALVES>
constexpr Launch few_gated() {
  if constexpr (BLOCKS % 2)
    return nullptr;  // (blocks of the gate and of the up come in pairs)
  else
    return launch_few<true, BLOCKS, TOKENS, WAVES, DEPTH, HALVES>;
}

// Fitted to 1000 sizes of 1-4096 tokens, 64-25600 features and columns, every variant with every
// split, plain and gated, weights read from memory.  The choice takes 1.018 times the fastest
// one's time on average (geometric mean; 1.07 in nine of ten sizes, 1.26 at worst).
#define FEW(B, T, W, D, H) \
  16 * B, T, 64 * W, W, H* FHALF, FewShape<B, T, W, D, H>::RINGS, B, true
#define TILE(TN, TM, WN, WM, ...) TN, TM, 64 * WN * WM, 0, 0, 0, 0, true
#define FEW_CALLS(B, T, W, D, H) {launch_few<false, B, T, W, D, H>, few_gated<B, T, W, D, H>()}
#define TILE_CALLS(...) {launch_tile<false, __VA_ARGS__>, launch_tile<true, __VA_ARGS__>}
constexpr Variant VARIANTS[] = {
    {FEW(1, 2, 4, 2, 2), 0, {2.639f, 0.091f, 0.f, 0.015f, 0.024f, 0.204f, 0.04f, 0.f, 0.f, 2.265f, 0.197f, 0.278f}, FEW_CALLS(1, 2, 4, 2, 2)},
    {FEW(2, 2, 4, 1, 2), 0, {2.689f, 0.233f, 0.f, 0.101f, 0.01f, 0.255f, 0.069f, 0.f, 0.f, 2.235f, 0.f, 0.275f}, FEW_CALLS(2, 2, 4, 1, 2)},
    {FEW(1, 4, 8, 2, 2), 0, {2.469f, 0.f, 0.f, 0.082f, 0.247f, 0.379f, 0.062f, 0.f, 0.f, 2.205f, 0.142f, 0.175f}, FEW_CALLS(1, 4, 8, 2, 2)},
    {FEW(2, 4, 4, 2, 2), 0, {2.807f, 0.01f, 0.082f, 0.007f, 0.f, 0.475f, 0.054f, 0.f, 0.f, 2.233f, 0.045f, 0.18f}, FEW_CALLS(2, 4, 4, 2, 2)},
    {FEW(2, 8, 4, 1, 2), 0, {2.773f, 0.21f, 0.f, 0.151f, 0.006f, 0.312f, 0.059f, 0.f, 0.f, 2.239f, 0.018f, 0.097f}, FEW_CALLS(2, 8, 4, 1, 2)},
    {FEW(2, 8, 8, 1, 1), 0, {2.743f, 0.074f, 0.f, 0.167f, 0.008f, 0.343f, 0.069f, 0.f, 0.f, 2.255f, 0.f, 0.143f}, FEW_CALLS(2, 8, 8, 1, 1)},
    {FEW(1, 16, 8, 2, 1), 0, {1.479f, 0.f, 0.f, 0.178f, 1.225f, 0.322f, 0.023f, 0.f, 0.f, 2.318f, 0.353f, 0.021f}, FEW_CALLS(1, 16, 8, 2, 1)},
    {FEW(2, 16, 8, 1, 1), 0, {2.712f, 0.025f, 0.f, 0.176f, 0.054f, 0.456f, 0.07f, 0.f, 0.f, 2.289f, 0.f, 0.023f}, FEW_CALLS(2, 16, 8, 1, 1)},
    {FEW(4, 16, 8, 1, 1), 0, {2.714f, 0.f, 0.053f, 0.231f, 0.176f, 0.78f, 0.086f, 0.f, 0.f, 2.219f, 0.f, 0.031f}, FEW_CALLS(4, 16, 8, 1, 1)},
    {FEW(2, 32, 8, 1, 1), 0, {1.303f, 0.f, 0.f, 0.249f, 1.664f, 0.636f, 0.066f, 0.f, 0.f, 2.385f, 0.f, 0.037f}, FEW_CALLS(2, 32, 8, 1, 1)},
    {FEW(4, 32, 4, 1, 1), 0, {3.06f, 0.153f, 0.f, 0.172f, 0.253f, 0.524f, 0.058f, 0.f, 0.f, 2.354f, 0.195f, 0.017f}, FEW_CALLS(4, 32, 4, 1, 1)},
    {FEW(4, 32, 8, 1, 1), 0, {1.2f, 0.f, 0.064f, 0.337f, 2.03f, 0.959f, 0.078f, 0.f, 0.f, 2.52f, 0.f, 0.043f}, FEW_CALLS(4, 32, 8, 1, 1)},
    {FEW(6, 32, 4, 1, 2), 0, {0.986f, 0.f, 0.703f, 0.088f, 2.74f, 1.856f, 0.083f, 0.f, 0.f, 2.809f, 0.095f, 0.02f}, FEW_CALLS(6, 32, 4, 1, 2)},
    {TILE(128, 32, 4, 1, 4, 3, true), 2, {1.862f, 0.014f, 0.172f, 0.045f, 0.479f, 0.02f, 0.093f, 0.982f, 0.194f, 2.32f, 0.226f, 0.f}, TILE_CALLS(128, 32, 4, 1, 4, 3, true)},
    {TILE(128, 64, 4, 1, 2, 2, false), 3, {2.782f, 0.f, 0.52f, 0.105f, 0.434f, 0.f, 0.092f, 0.f, 0.375f, 1.872f, 0.302f, 0.f}, TILE_CALLS(128, 64, 4, 1, 2, 2, false)},
    {TILE(256, 64, 8, 1, 4, 3, true), 0, {1.715f, 0.f, 1.17f, 0.081f, 2.407f, 0.391f, 0.057f, 0.f, 0.f, 2.363f, 0.265f, 0.f}, TILE_CALLS(256, 64, 8, 1, 4, 3, true)},
    {TILE(256, 128, 8, 1, 4, 3, false), 0, {1.981f, 0.f, 2.306f, 0.187f, 2.833f, 0.605f, 0.006f, 0.f, 0.f, 2.407f, 0.235f, 0.f}, TILE_CALLS(256, 128, 8, 1, 4, 3, false)},
    {TILE(256, 256, 8, 1, 2, 2, false), 0, {3.25f, 0.f, 4.988f, 0.334f, 2.831f, 1.111f, 0.004f, 0.f, 0.f, 3.23f, 0.171f, 0.f}, TILE_CALLS(256, 256, 8, 1, 2, 2, false)},
};
#undef FEW
#undef TILE
#undef FEW_CALLS
#undef TILE_CALLS

int64_t weight_bytes(bool gated, int n, int k) {
  return (int64_t)n * k / 32 * (gated ? 34 : 17);
}

template <bool GATED>
int launch(dlfp::ProjectionArgs& a, void* workspace, size_t bytes, hipStream_t stream) {
  (void)hipGetLastError();
  if (std::max<int64_t>(a.ldx, a.k) >= FAR_STRIDE) return launch_far<GATED>(a, stream);
  return launch_best(VARIANTS, GATED, a, weight_bytes(GATED, a.n, a.k), workspace, bytes, stream);
}

}  // namespace

namespace dlfp {

int check_projection(ProjectionArgs& a, bool gated, bool codes, int32_t out_dtype,
                     const void* workspace) {
  if (a.m < 0 || a.n <= 0 || a.k <= 0) return DLFP_EINVAL;
  if (out_dtype != 0 && out_dtype != 1) return DLFP_EINVAL;
  if (gated && a.act != DLFP_SILU && a.act != DLFP_GELU) return DLFP_EINVAL;
  if (a.n % 16 || a.k % 64) return DLFP_EUNSUPPORTED;
  if (a.ldx < a.k || a.ldo < a.n || a.ldx % 8 || a.ldo % 4) return DLFP_EINVAL;
  if (too_many(a.m, a.n)) return DLFP_ERANGE;
  if (a.m == 0) return DLFP_OK;
  const auto aligned = [](const void* p, uintptr_t to) {
    return p && reinterpret_cast<uintptr_t>(p) % to == 0;
  };
  if (!aligned(a.x, 16) || !aligned(a.out, out_dtype ? 16 : 8)) return DLFP_EINVAL;
  if (workspace && !aligned(workspace, 16)) return DLFP_EINVAL;
  for (int i = 0; i < (gated ? 2 : 1); ++i) {
    if (!aligned(a.weights[i], 16)) return DLFP_EINVAL;
    if (codes && !aligned(a.exps[i], 16)) return DLFP_EINVAL;
  }
  a.wide = aligned(a.out, 16) && a.ldo % 8 == 0;
  return DLFP_OK;
}

}  // namespace dlfp

extern "C" int dlfp_linear_w4(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                              const void* codes, const void* exps, void* out, int64_t ldo,
                              int32_t out_dtype, void* workspace, size_t workspace_bytes,
                              hipStream_t stream) {
  dlfp::ProjectionArgs a{static_cast<const uint16_t*>(x),
                         {codes, nullptr},
                         m, n, k, 0, ldx, ldo, out,
                         {static_cast<const uint8_t*>(exps), nullptr},
                         out_dtype, 0, 0};
  const int st = dlfp::check_projection(a, false, true, out_dtype, workspace);
  return st != DLFP_OK || m == 0 ? st : launch<false>(a, workspace, workspace_bytes, stream);
}

extern "C" int dlfp_gated_linear_w4(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                                    const void* gate_codes, const void* gate_exps,
                                    const void* up_codes, const void* up_exps, int32_t activation,
                                    void* out, int64_t ldo, int32_t out_dtype, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream) {
  dlfp::ProjectionArgs a{
      static_cast<const uint16_t*>(x),
      {gate_codes, up_codes},
      m, n, k, activation, ldx, ldo, out,
      {static_cast<const uint8_t*>(gate_exps), static_cast<const uint8_t*>(up_exps)},
      out_dtype, 0, 0};
  const int st = dlfp::check_projection(a, true, true, out_dtype, workspace);
  return st != DLFP_OK || m == 0 ? st : launch<true>(a, workspace, workspace_bytes, stream);
}

namespace dlfp {

Form form_w4(bool gated, int m, int n, int k, int64_t room) {
  return form_of(VARIANTS, gated, m, n, k, weight_bytes(gated, n, k), room);
}

namespace {

// DLFP_OK and the form of a call of near rows, or what is wrong with the sizes.
int form_of_kind(int32_t kind, int32_t m, int32_t n, int32_t k, size_t bytes, Form& form) {
  if (kind < DLFP_LINEAR_W4 || kind > DLFP_GATED_LINEAR_W4) return DLFP_EINVAL;
  if (m <= 0 || n <= 0 || k <= 0) return DLFP_EINVAL;
  if (n % 16 || k % 64) return DLFP_EUNSUPPORTED;
  if (k >= FAR_STRIDE || too_many(m, n)) return DLFP_ERANGE;
  const int64_t room = (int64_t)std::min<size_t>(bytes, MOST_PARTS);
  form = kind == DLFP_GATED_LINEAR_BF16 ? form_gated(m, n, k, room)
                                        : form_w4(kind == DLFP_GATED_LINEAR_W4, m, n, k, room);
  return form.variant < 0 ? DLFP_ERANGE : DLFP_OK;
}

}  // namespace

}  // namespace dlfp

extern "C" int64_t dlfp_projection_workspace(int32_t kind, int32_t m, int32_t n, int32_t k) {
  dlfp::Form form;
  return dlfp::form_of_kind(kind, m, n, k, SIZE_MAX, form) == DLFP_OK ? form.bytes : 0;
}

extern "C" int dlfp_projection_form_of(int32_t kind, int32_t m, int32_t n, int32_t k,
                                       size_t workspace_bytes, dlfp_projection_form* form) {
  if (!form) return DLFP_EINVAL;
  dlfp::Form f;
  const int st = dlfp::form_of_kind(kind, m, n, k, workspace_bytes, f);
  if (st == DLFP_OK) *form = {f.variant, f.rows, f.tokens, f.splits, f.stream, 0, f.bytes};
  return st;
}
