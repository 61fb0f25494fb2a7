// Paged KV append into 8-bit pages, with the position rotation on the way
// (dlfp_rope_append_kv8; the page format is declared in dlfp_cache.h).
//
// The new tokens of one page are one "run": consecutive rows with consecutive
// slots, at most 16.  A wavefront takes a run of one KV head: it holds the run's
// keys and values in registers (eight dims of four tokens to a lane: 16 lanes a
// row), finds their largest magnitude, from it and the page's exponent the new
// exponent, and stores the codes.  Because the exponent of a page belongs to all
// its tokens, a page is never written by two wavefronts, and the older tokens'
// codes are rewritten by the same wavefront when the exponent grows: their values
// stay as they are but for codes that become subnormal (power-of-two scales).
//
// A key row of codes is 128 bytes, 8 to a lane.  A value row (one dimension, 16
// slots) is 16 bytes: the four tokens' codes of a dimension meet through LDS,
// which holds the page's 2 KiB as it is stored, so that values go out as whole
// kilobytes; of a page that is not written from slot 0 to 15, the rows are read
// first and put back with the other slots' codes as they were.
//
// Bound by its chain of round trips (slots, tokens and page, codes: 4.2 us from one
// token to 64 decoders) up to some 500 tokens and by its bytes from there: with 64
// and 8 heads 256 decoders 6.4 us, 2048 tokens 17.9 (81 MB, 4.5 TB/s), 8192 tokens
// 68 (323 MB, 4.75 TB/s, the rate of a copy).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "dlfp_cache.h"
#include "dlfp_internal.h"
#include "rope_device.h"

namespace {

constexpr int D = DLFP_HEAD_DIM;
constexpr int PAGE = DLFP_PAGE_SIZE;
constexpr int PAGE_BYTES = PAGE * D;
constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;
constexpr int EXP_MIN = -100, EXP_BIAS = 127;

struct Args {
  RopeArgs rope;
  QueryArgs query;
  const int32_t* positions;
  const int32_t* slots;
  const uint16_t* k_new;
  const uint16_t* v_new;
  int64_t ldk, ldv;
  uint8_t* k_cache;
  uint8_t* v_cache;
  uint8_t* k_exp;
  uint8_t* v_exp;
  int num_tokens;
  int hkv;
  int64_t num_slots;
  int window;   // tokens of a workgroup: 4 or 16
  int blocks;   // workgroups of a KV head
};

// Position of token slot t inside a value page row (bits 2 and 3 swap).
__device__ __forceinline__ int vt_pos(int t) { return (t & 3) | ((t & 4) << 1) | ((t & 8) >> 1); }

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

// Magnitude for the page's exponent: NaN and infinities do not count.
__device__ __forceinline__ float magnitude(float x) {
  const float m = __builtin_fabsf(x);
  return m < __builtin_inff() ? m : 0.f;
}

// The least E >= EXP_MIN with amax <= 448 * 2^E: with amax = m 2^x, 1 <= m < 2,
// and 448 = 1.75 * 2^8 that is x - 8, or x - 7 when m > 1.75.  (Subnormal amax:
// x reads as -127, far below EXP_MIN either way.)
__device__ __forceinline__ int page_exponent(float amax) {
  const uint32_t b = __builtin_bit_cast(uint32_t, amax);
  const int x = (int)(b >> 23) - 127;
  return max(EXP_MIN, x - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}
__device__ __forceinline__ float power2(int e) {  // -126 <= e <= 127
  return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}
// A multiplication by 2^e for any e that a page's exponents can be apart.
__device__ __forceinline__ float scaled(float x, int e) { return __builtin_ldexpf(x, e); }

// Four values into four codes (round to nearest even; |x| <= 448, or NaN).
__device__ __forceinline__ uint32_t codes(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
// What a page cannot hold becomes NaN (an infinity; the scale covers the rest).
__device__ __forceinline__ float held(float x) {
  return __builtin_fabsf(x) < __builtin_inff() ? x : __builtin_nanf("");
}
// Four codes whose exponent grows by `up`.
__device__ __forceinline__ uint32_t moved(uint32_t w, int up) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  return codes(scaled(lo[0], -up), scaled(lo[1], -up), scaled(hi[0], -up), scaled(hi[1], -up));
}

// Where a value row (16 bytes) sits in LDS: rows 8 c + x of the 16 chunks c, which
// the lanes write together, fall on different banks.
__device__ __forceinline__ int lds_row(int d) { return d ^ ((d >> 4) & 7); }

// Lanes of one wavefront hand data to each other through LDS (and, between the
// runs of one page, through memory).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The run of tokens first .. first + n - 1 from slot o0 of a page, one KV head.
// lds: 2 KiB of the wavefront's own.
__device__ void append_run(const Args& a, int first, int n, int slot0, int h, uint8_t* lds) {
  const int lane = threadIdx.x & 63, chunk = lane & 15, quarter = lane >> 4;
  const int o0 = slot0 & (PAGE - 1);
  const int64_t page = (int64_t)(slot0 >> 4) * a.hkv + h;
  uint8_t* kp = a.k_cache + page * PAGE_BYTES;
  uint8_t* vp = a.v_cache + page * PAGE_BYTES;

  // Token 4 j + quarter of the run in kx[j], vx[j]; past its end the last one
  // again, which changes no maximum and is not stored.
  uint4 kx[4], vx[4];
  int pos[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (4 * j >= n) break;
    const int64_t t = first + min(4 * j + quarter, n - 1);
    pos[j] = a.positions[t];
    kx[j] = *reinterpret_cast<const uint4*>(a.k_new + t * a.ldk + h * D + 8 * chunk);
    vx[j] = *reinterpret_cast<const uint4*>(a.v_new + t * a.ldv + h * D + 8 * chunk);
  }
  const bool whole = n == PAGE;
  const int k_was = a.k_exp[page], v_was = a.v_exp[page];
  // Value rows 2 lane and 2 lane + 1 as they are, 32 bytes.
  uint4 rows[2] = {};
  if (!whole) {
    rows[0] = reinterpret_cast<const uint4*>(vp)[2 * lane];
    rows[1] = reinterpret_cast<const uint4*>(vp)[2 * lane + 1];
  }
  float y[4][8];
  float k_max = 0.f, v_max = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (4 * j >= n) break;
    const uint32_t x[4] = {kx[j].x, kx[j].y, kx[j].z, kx[j].w};
    rotate(a.rope, load_turn(a.rope, pos[j], chunk), chunk, x, y[j]);
    const uint32_t v[4] = {vx[j].x, vx[j].y, vx[j].z, vx[j].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) k_max = fmaxf(k_max, magnitude(y[j][i]));
#pragma unroll
    for (int w = 0; w < 4; ++w)
      v_max = fmaxf(v_max, fmaxf(magnitude(__builtin_bit_cast(float, v[w] << 16)),
                                 magnitude(__builtin_bit_cast(float, v[w] & 0xFFFF0000u))));
  }
  int k_e = page_exponent(wave_max(k_max)), v_e = page_exponent(wave_max(v_max));
  if (o0 > 0) {
    k_e = max(k_e, k_was - EXP_BIAS);
    v_e = max(v_e, v_was - EXP_BIAS);
  }

  // Keys: the older rows first if their exponent grows, then the new ones.
  if (o0 > 0 && k_e > k_was - EXP_BIAS) {
    const int up = k_e - (k_was - EXP_BIAS);
    for (int r = lane >> 3; r < o0; r += 8) {
      uint4* p = reinterpret_cast<uint4*>(kp + r * D) + (lane & 7);
      uint4 w = *p;
      w.x = moved(w.x, up), w.y = moved(w.y, up), w.z = moved(w.z, up), w.w = moved(w.w, up);
      *p = w;
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (4 * j >= n) break;
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = held(scaled(y[j][i], -k_e));
    const uint2 c = {codes(z[0], z[1], z[2], z[3]), codes(z[4], z[5], z[6], z[7])};
    const int i = 4 * j + quarter;
    if (i < n) *reinterpret_cast<uint2*>(kp + (o0 + i) * D + 8 * chunk) = c;
  }

  // Values: the rows as they are to LDS, the older slots' codes moved; the new
  // codes into their bytes; the rows out again.
  if (!whole) {
    const int up = o0 > 0 ? v_e - (v_was - EXP_BIAS) : 0;
    if (up > 0) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&rows[r]);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          // word x holds positions 4 x .. 4 x + 3: slots vt_pos(4 x) .. + 3
          const int older = min(max(o0 - vt_pos(4 * x), 0), 4);
          const uint32_t mask = older == 4 ? ~0u : (1u << (8 * older)) - 1;
          w[x] = (moved(w[x], up) & mask) | (w[x] & ~mask);
        }
      }
    }
    reinterpret_cast<uint4*>(lds)[lds_row(2 * lane)] = rows[0];
    reinterpret_cast<uint4*>(lds)[lds_row(2 * lane + 1)] = rows[1];
  }
  wave_fence();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (4 * j >= n) break;
    const uint32_t v[4] = {vx[j].x, vx[j].y, vx[j].z, vx[j].w};
    uint32_t c[2];
#pragma unroll
    for (int w = 0; w < 2; ++w)
      c[w] = codes(held(scaled(__builtin_bit_cast(float, v[2 * w] << 16), -v_e)),
                   held(scaled(__builtin_bit_cast(float, v[2 * w] & 0xFFFF0000u), -v_e)),
                   held(scaled(__builtin_bit_cast(float, v[2 * w + 1] << 16), -v_e)),
                   held(scaled(__builtin_bit_cast(float, v[2 * w + 1] & 0xFFFF0000u), -v_e)));
    const int i = 4 * j + quarter;
    if (i < n) {
      uint8_t* at = lds + vt_pos(o0 + i);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        at[lds_row(8 * chunk + x) * PAGE] = (uint8_t)(c[x >> 2] >> (8 * (x & 3)));
    }
  }
  wave_fence();
#pragma unroll
  for (int r = 0; r < 2; ++r)
    reinterpret_cast<uint4*>(vp)[64 * r + lane] =
        reinterpret_cast<const uint4*>(lds)[lds_row(64 * r + lane)];
  if (lane == 0) {
    a.k_exp[page] = (uint8_t)(k_e + EXP_BIAS);
    a.v_exp[page] = (uint8_t)(v_e + EXP_BIAS);
  }
  // The next run may be one of the same page, and fills lds after these reads.
  wave_fence();
}

// Workgroups: for each KV head and window of tokens the runs that begin there, in
// turn over the wavefronts; then the queries.
__global__ __launch_bounds__(THREADS) void kv8_append_kernel(const Args a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[WAVES][PAGE_BYTES];
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  int block = blockIdx.x;
  if (block >= a.blocks * a.hkv) {
    const int item = (block - a.blocks * a.hkv) * WAVES + wave;
    if (item < a.num_tokens * a.query.chunks) rotate_queries(a.query, a.rope, a.positions, item);
    return;
  }
  const int h = block / a.blocks;
  block -= h * a.blocks;
  const int t0 = block * a.window, t1 = min(t0 + a.window, a.num_tokens);
  // Lane l has the slot of token t0 - 16 + l: the 16 before the window's (at most
  // 16), and the 15 after.
  const int t = t0 - PAGE + lane;
  const bool real = t >= 0 && t < a.num_tokens && lane < a.window + 2 * PAGE;
  int slot = real ? a.slots[t] : -1;
  const int pos = real ? a.positions[t] : -1;
  if ((unsigned)pos >= (unsigned)a.rope.positions || (int64_t)slot >= a.num_slots) slot = -1;
  // A token goes on with the run of the one before when its slot follows in the
  // same page; a run joins the one before (tokens left out between them do not
  // count) when it goes on in the same page: one wavefront then takes both.
  const uint64_t valid = __builtin_amdgcn_ballot_w64(slot >= 0);
  const int before = __shfl_up(slot, 1);
  const bool follows = lane > 0 && slot > 0 && slot == before + 1 && (slot & (PAGE - 1)) != 0;
  const uint64_t goes_on = __builtin_amdgcn_ballot_w64(follows);
  const uint64_t lower = valid & ((1ull << lane) - 1);
  const int last = __shfl(slot, lower ? 63 - __builtin_clzll(lower) : 0);
  const uint64_t starts = valid & ~goes_on;
  const uint64_t joins = starts & __builtin_amdgcn_ballot_w64(lower != 0 && last < slot &&
                                                              last >> 4 == slot >> 4);
  uint64_t begins = starts & ~joins & (((1ull << (t1 - t0)) - 1) << PAGE);
  for (int i = 0; begins; ++i, begins &= begins - 1) {
    if (i % WAVES != wave) continue;
    for (int l = __builtin_ctzll(begins);;) {
      const int n = 1 + __builtin_ctzll(~(goes_on >> (l + 1)));
      append_run(a, t0 - PAGE + l, n, __builtin_amdgcn_readlane(slot, l), h, lds[wave]);
      const uint64_t rest = starts & ~((2ull << l) - 1);
      l = rest ? __builtin_ctzll(rest) : 0;
      if (!(joins >> l & 1) || !rest) break;
    }
  }
}

}  // namespace

extern "C" int dlfp_rope_append_kv8(const dlfp_dims* dims, const dlfp_rope* rope,
                                    int32_t num_tokens, const int32_t* positions,
                                    const int32_t* slot_mapping, const void* q, int64_t ldq,
                                    const void* k_new, int64_t ldk, const void* v_new, int64_t ldv,
                                    void* q_out, int64_t ldo, void* k_cache, void* v_cache,
                                    uint8_t* k_exp, uint8_t* v_exp, int32_t num_blocks,
                                    hipStream_t stream) {
  const int st = dlfp::check_rope_append(dims, rope, num_tokens, positions, slot_mapping, q, ldq,
                                         k_new, ldk, v_new, ldv, q_out, ldo, k_cache, v_cache,
                                         num_blocks);
  if (st != DLFP_OK || num_tokens == 0) return st;
  if (!k_exp || !v_exp) return DLFP_EINVAL;
  Args a;
  a.rope = {rope->table, rope->positions, rope->rotary_dim, rope->interleaved};
  a.query = {static_cast<const uint16_t*>(q), static_cast<uint16_t*>(q_out), ldq, ldo,
             dims->num_q_heads, 0};
  a.positions = positions;
  a.slots = slot_mapping;
  a.k_new = static_cast<const uint16_t*>(k_new);
  a.v_new = static_cast<const uint16_t*>(v_new);
  a.ldk = ldk;
  a.ldv = ldv;
  a.k_cache = static_cast<uint8_t*>(k_cache);
  a.v_cache = static_cast<uint8_t*>(v_cache);
  a.k_exp = k_exp;
  a.v_exp = v_exp;
  a.num_tokens = num_tokens;
  a.hkv = dims->num_kv_heads;
  a.num_slots = (int64_t)num_blocks * PAGE;
  a.query.chunks = query_chunks(dims->num_q_heads);
  // A window of 4 tokens for 4 wavefronts gives each run of a decoder, a token, a
  // wavefront to itself; of a prompt's chunk, where a run begins every 16 tokens, most
  // windows begin none and their workgroups cost their launch.  With windows of 4 and
  // of 16, 64 and 8 heads: 64 decoders 4.5 and 9.3 us, 256 6.4 and 11.1, 1024 17.3 and
  // 17.3, 2048 36 and 32; a chunk of 512 tokens 9.6 and 8.7, of 1024 14.6 and 11.3, of
  // 8192 107 and 68.
  a.window = num_tokens <= 512 ? 4 : 16;
  a.blocks = (num_tokens + a.window - 1) / a.window;
  const int64_t queries = ((int64_t)num_tokens * a.query.chunks + WAVES - 1) / WAVES;
  (void)hipGetLastError();
  kv8_append_kernel<<<(unsigned)((int64_t)a.blocks * a.hkv + queries), THREADS, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? DLFP_OK : DLFP_EHIP;
}
