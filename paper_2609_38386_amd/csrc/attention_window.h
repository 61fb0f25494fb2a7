// Paged attention with a sliding window and sinks, over bf16 or 8-bit pages: the
// kernels of dlfp_attention_window and dlfp_attention_kv8, which differ in how a
// page reaches the matrix products (template parameter KV8).
//
// A row at position p sees key j <= p with p - j < window or j < sinks.  A unit
// (the rows of one tile of a prompt, or one decoding token, for one KV head)
// reads only pages that hold a key some row of it sees: its sink pages, then,
// past a gap of whole pages, those from its first row's window on.  Work records
// count keys without the gap ("virtual" keys, whole pages), so a unit is a range
// [KVBEGIN, KVEND) of them whatever the mask, and a unit's table of block ids in
// LDS lists its pages in that order; only masks go back to positions.
//
// 8-bit pages travel to LDS as they are stored, by direct copies, half the bytes.
// With a power of two as a page's scale, v_cvt_scalef32_pk_bf16_fp8 turns two codes
// into the two bf16 numbers that they stand for, so that values, and with fp32
// output keys, are operands of the same bf16 products from there on: 16 codes (one
// 16-byte LDS read) make two operands of eight.  Which dims and keys a lane's eight
// are is free as long as both factors of a product agree, so a lane takes 16 codes
// that are next to each other: of a key row, dims 32 j + 16 hi .. + 15 (of 32 x 32
// products; of 16 x 16 ones 64 j + 16 q ..); of a value row, all 16 slots of one page.
// With bf16 output keys are not converted: a query is a sum of two rows of codes, and
// scores are products of codes with the pages' exponents as their block scales, twice
// the bf16 rate for twice the products, without the conversions (prompts of 1999
// tokens over 8144 keys 445 -> 396 us).
//
// Everything else is as in attention_mixed.hip: S^T = K Q^T and O^T += V^T P^T
// with row statistics in a lane, a lazily raised reference maximum in the exp2
// domain, split ranges merged by the last to finish.
#ifndef DLFP_ATTENTION_WINDOW_H
#define DLFP_ATTENTION_WINDOW_H

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "attention_device.h"
#include "dlfp_cache.h"
#include "dlfp_internal.h"

namespace {

constexpr int KV_TILE = 64;  // keys per prefill tile (4 pages)
constexpr int THREADS = 256;
constexpr int SMALL_ROWS = DLFP_SMALL_ROWS;  // units of at most so many rows split their keys
constexpr int PRE_PTAB = DLFP_MAX_PREFILL_UNIT_KEYS / PAGE;
constexpr int DEC_PTAB = DLFP_MAX_DECODE_UNIT_KEYS / PAGE;

struct Args {
  const int32_t* work;
  const int32_t* block_table;
  const uint16_t* q;
  const char* kc;
  const char* vc;
  const uint8_t* k_exp;  // 8-bit pages only
  const uint8_t* v_exp;
  void* out;
  float* ws;
  int32_t max_blocks;
  int32_t num_blocks;
  int32_t hq;
  int32_t hkv;
  int32_t num_units;
  int32_t num_prefill;
  int32_t out_f32;
  // Grid of a launch with both shares: `lead` prefill workgroups, `decode_lead`
  // decode ones, then either `decode_rest` more and the other prefill ones, or groups
  // of GRID_GROUP workgroups, prefill_groups and decode_groups of them evenly mixed,
  // and what is left of each share.
  int32_t lead, decode_lead, decode_rest, prefill_groups, decode_groups;
  int32_t solo;  // a decode workgroup has four units, a wavefront each
  float scale_log2;
};

// Bytes of a (block, head) page of keys or values.
template <bool KV8>
constexpr int page_bytes() {
  return KV8 ? PAGE_ELEMS : 2 * PAGE_ELEMS;
}

// Two bf16 operands from 16 codes of a page whose scale is `scale`.
typedef uint32_t codes_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void widen(codes_t c, float scale, bf16x8_t* lo, bf16x8_t* hi) {
  u32x4_t a, b;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    a[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[w], scale, false));
    a[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[w], scale, true));
    b[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[w + 2], scale, false));
    b[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[w + 2], scale, true));
  }
  *lo = __builtin_bit_cast(bf16x8_t, a);
  *hi = __builtin_bit_cast(bf16x8_t, b);
}
// The scale of an exponent byte (0: 2^-127, a subnormal; 255: infinity, NaN out).
__device__ __forceinline__ float scale_of(int byte) {
  return __builtin_bit_cast(float, byte ? (uint32_t)byte << 23 : 0x00400000u);
}

// Codes of 16-byte pieces as the operand of a product of 8-bit numbers.
typedef int operand8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ operand8_t operand8(codes_t a, codes_t b) {
  operand8_t x;
#pragma unroll
  for (int w = 0; w < 4; ++w) x[w] = (int)a[w], x[w + 4] = (int)b[w];
  return x;
}
// Four numbers into the codes nearest to x / scale, and two codes back times scale.
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d, float scale) {
  typedef short s16x2_t __attribute__((ext_vector_type(2)));
  s16x2_t x = {0, 0};
  x = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x, a, b, scale, false);
  x = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, x);
}

// A query row for products with keys of codes: a bf16 number is a sum of two e4m3
// codes (4 bits each) in scales 2^4 apart, exactly but for numbers below 2^-14 of
// the row's largest, which lose what lies below 2^-22 of it.  x: the lane's dims
// (eight to a word group), amax: the row's largest magnitude.  hi and lo: the
// codes; returns the exponent byte of hi's scale, lo's is 4 less.
__device__ __forceinline__ float largest(bf16x8_t x) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, __builtin_fabsf((float)x[i]));
  return m;
}
__device__ __forceinline__ int row_exponent(float amax) {  // amax <= 448 * 2^(e - 127)
  return max(27, (int)(__builtin_bit_cast(uint32_t, amax) >> 23) - 7);
}
__device__ __forceinline__ void split_codes(bf16x8_t x, int e, uint32_t* hi, uint32_t* lo) {
  const float s = scale_of(e), t = scale_of(e - 4);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)x[4 * w + i];
    hi[w] = to_codes(f[0], f[1], f[2], f[3], s);
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi[w], s, false);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi[w], s, true);
    lo[w] = to_codes(f[0] - a[0], f[1] - a[1], f[2] - b[0], f[3] - b[1], t);
  }
}

// The codes of a row of 32 x 32 products, whose dims two lanes hold 16 by 16:
// q8[high, low term][dims 64 d .. + 63].  Returns the exponent byte.
__device__ __forceinline__ int query_codes(const bf16x8_t* q, operand8_t (*q8)[2]) {
  float m = 0.f;
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) m = fmaxf(m, largest(q[kk]));
  const int e = row_exponent(max_xor32(m));
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) {
    uint32_t hi[2], lo[2];
    split_codes(q[kk], e, hi, lo);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      q8[0][kk >> 2][2 * (kk & 3) + w] = (int)hi[w];
      q8[1][kk >> 2][2 * (kk & 3) + w] = (int)lo[w];
    }
  }
  return e;
}

// Which keys a unit's rows see, in virtual keys: a row at position p those below
// end(p) that are not below low(p), or are below `sinks`.  (The gap ends before
// the window of every row of the unit, so the sink pages keep their positions and
// all other keys move by the gap.)
struct Span {
  int window, sinks;
  int sink_pages, gap;  // virtual pages from sink_pages on are `gap` pages further
  __device__ __forceinline__ int page(int vp) const { return vp >= sink_pages ? vp + gap : vp; }
  __device__ __forceinline__ int low(int p) const { return max(p - window + 1 - PAGE * gap, 0); }
  __device__ __forceinline__ int end(int p) const { return p + 1 - PAGE * gap; }
  // Whether virtual keys [v0, v1) hold one that rows up to position p do not see
  // because it lies before their window.
  __device__ __forceinline__ bool below(int v0, int v1, int p) const {
    return v0 < low(p) && v1 > sinks;
  }
  // Bit i: the position of the value page from virtual key v on whose slot is seen
  // by a row at p, keys from `stop` on left out.
  __device__ __forceinline__ uint32_t seen(int v, int p, int stop) const {
    auto first = [](int n) { return (1u << min(max(n, 0), PAGE)) - 1; };
    const uint32_t m = (~first(low(p) - v) | first(sinks - v)) & first(stop - v);
    return (m & 0xF00Fu) | ((m & 0x00F0u) << 4) | ((m & 0x0F00u) >> 4);
  }
};
__device__ __forceinline__ Span span_of(record_t f) {
  Span s;
  s.window = f[DLFP_W_WINDOW];
  s.sinks = f[DLFP_W_SINKS];
  s.gap = f[DLFP_W_GAP];
  s.sink_pages = s.gap ? (s.sinks + PAGE - 1) / PAGE : 0;
  return s;
}
// Masks of a pair of 16-bit values, of four bytes, from their bits.
__device__ __forceinline__ uint32_t pair_mask(uint32_t bits) {
  return (bits & 1 ? 0x0000FFFFu : 0u) | (bits & 2 ? 0xFFFF0000u : 0u);
}
__device__ __forceinline__ uint32_t byte_mask(uint32_t bits) {
  return (((bits & 15) * 0x00204081u) & 0x01010101u) * 0xFFu;
}

// The values of a word (four codes, two bf16 numbers) that are infinite or NaN.
template <bool KV8>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  if constexpr (KV8) return ((((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xFFu;
  return ((((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xFFFFu;
}

// Zeroes in LDS the values of BP pages from virtual key v0 on that a row at `pos`
// does not see, or that lie at or past `stop` (one wavefront).  FINITE: also those
// that are infinite or NaN.
template <bool KV8, int BP, bool FINITE>
__device__ __forceinline__ void zero_values(char* values, const Span& sp, int v0, int pos,
                                            int stop) {
  constexpr int PB = page_bytes<KV8>();
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int pg = 0; pg < BP; ++pg) {
    const uint32_t seen = sp.seen(v0 + pg * PAGE, pos, stop);
    if (!FINITE && seen == 0xFFFFu) continue;
    u32x4_t* page = reinterpret_cast<u32x4_t*>(values + pg * PB);
#pragma unroll
    for (int c = 0; c < PB / 1024; ++c) {
      const int ck = 64 * c + lane;
      u32x4_t v = page[ck];
      if constexpr (KV8) {
#pragma unroll
        for (int w = 0; w < 4; ++w) v[w] &= byte_mask(seen >> (4 * w));
      } else {
        const bool upper = (ck & 1) ^ vt_swz(ck >> 1);  // positions 8 .. 15
#pragma unroll
        for (int w = 0; w < 4; ++w)
          v[w] &= upper ? pair_mask(seen >> (8 + 2 * w)) : pair_mask(seen >> (2 * w));
      }
      if constexpr (FINITE) {
#pragma unroll
        for (int w = 0; w < 4; ++w) v[w] &= ~not_finite<KV8>(v[w]);
      }
      page[ck] = v;
    }
  }
}

// Probabilities of two keys as bf16 pairs, for the matrix products.  bf16 output:
// one term, rounded to nearest: 1.1e-3 to 1.6e-3 of a row in the 2-norm, below
// what rounding the output leaves (1.7e-3).  fp32 output: three terms, the first
// two cut off so that none is negative, 24 bits together.
__device__ __forceinline__ uint32_t cut(float& a, float& b) {
  const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
  a -= __builtin_bit_cast(float, x & 0xFFFF0000u);
  b -= __builtin_bit_cast(float, y & 0xFFFF0000u);
  return __builtin_amdgcn_perm(y, x, 0x07060302u);
}
// A later term, at least the least normal number where the term before is one too
// (8-bit pages hold no infinity): a term of 0 would make a NaN of an infinite value
// that the row sees, and one above 0 would give a masked key a weight.
template <bool KV8>
__device__ __forceinline__ uint32_t above_zero(uint32_t term, uint32_t before) {
  if constexpr (KV8) return term;
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
  const u16x2_t least = {0x0080, 0x0080};
  const u16x2_t floor = __builtin_elementwise_min(__builtin_bit_cast(u16x2_t, before), least);
  return __builtin_bit_cast(
      uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, term), floor));
}

// Values that are not finite of keys that some rows of a unit see and others do not: a
// probability of 0 times one is NaN.  A prompt's unit whose sums are not all finite does
// its work again with such values as zero in the tiles that not all rows see whole, and
// then adds what they are to the results that one reaches: for each 32 rows (`first`
// and on) and such a tile of `tile` keys, it multiplies what a value is, a digit of a
// count for each kind, with 1 where a row sees the key, else 0.  (Zeroed as tiles come
// in, the same costs all prompts 1% to 6%; so it is a look at a unit's sums, 0.2% of long
// prompts and 1% of short ones, and up to twice the time where all units meet one.)
__device__ __forceinline__ bool all_finite(const f32x16_t* o) {
  uint32_t most = 0;
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const float y = o[mb][x];  // (a bit cast of the element itself reads element 0)
      most = max(most, __builtin_bit_cast(uint32_t, y) & 0x7FFFFFFFu);
    }
  return most < 0x7F800000u;
}
__device__ __forceinline__ bf16x8_t kinds_of(bf16x8_t values) {
  u32x4_t v = __builtin_bit_cast(u32x4_t, values);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t kind = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t x = v[w] >> (16 * h) & 0xFFFFu;
      const uint32_t k = (x & 0x7FFFu) > 0x7F80u ? 0x4980u    // NaN: 2^20
                         : x == 0x7F80u          ? 0x3F80u    // infinity: 1
                         : x == 0xFF80u          ? 0x4480u    // -infinity: 2^10
                                                 : 0u;
      kind |= k << (16 * h);
    }
    v[w] = kind;
  }
  return __builtin_bit_cast(bf16x8_t, v);
}
template <int G, bool KV8>
__device__ __forceinline__ void add_special(const Args& a, const record_t f, int first, int tile) {
  constexpr int PB = page_bytes<KV8>();
  const int lane = threadIdx.x & 63, col = lane & 31, hi = lane >> 5;
  const int kh = f[DLFP_W_KVHEAD], nt = f[DLFP_W_QNTOK];
  const int vb = f[DLFP_W_KVBEGIN], ve = f[DLFP_W_KVEND], nsplits = f[DLFP_W_NSPLITS];
  const Span sp = span_of(f);
  const int32_t* bt = a.block_table + (int64_t)f[DLFP_W_SEQ] * a.max_blocks;
  const int r = first + col, tr = r / G;
  const bool row_ok = tr < nt;
  const int end = row_ok ? min(sp.end(f[DLFP_W_QPOS0] + tr), ve) : 0;
  const int low = row_ok ? sp.low(f[DLFP_W_QPOS0] + tr) : 0;
  const int last_page = (ve - 1) / PAGE;
  const int unit_end = min(sp.end(f[DLFP_W_QPOS0]), ve), last = f[DLFP_W_QPOS0] + nt - 1;

  f32x16_t o[4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) o[mb] = f32x16_t{};
  for (int v0 = vb; v0 < ve; v0 += 2 * PAGE) {
    const int t0 = v0 - (v0 - vb) % tile;
    if (t0 + tile <= unit_end && !sp.below(t0, t0 + tile, last)) continue;
    // Step h: 16 keys, in the order of the probabilities of the units (of 8-bit pages
    // this lane has eight of page hi).
    bf16x8_t sees[2];
    const char* page[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4_t w = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int x = 8 * h + e;
        const int key = v0 + (KV8 ? 16 * hi + vt_pos(x) : 4 * hi + 8 * (x >> 2) + (x & 3));
        if (key < end && (key >= low || key < sp.sinks)) w[e >> 1] |= 0x3F80u << (16 * (e & 1));
      }
      sees[h] = __builtin_bit_cast(bf16x8_t, w);
      const int id = bt[sp.page(min(v0 / PAGE + (KV8 ? hi : h), last_page))];
      const int64_t block = (unsigned)id < (unsigned)a.num_blocks ? id : 0;
      page[h] = a.vc + (block * a.hkv + kh) * PB + (KV8 ? 0 : 16 * hi);
    }
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) {
      const int d = (32 * mb + col) * (PB / D);
      bf16x8_t v[2];
      if constexpr (KV8) {
        widen(*reinterpret_cast<const codes_t*>(page[0] + d), 1.f, &v[0], &v[1]);
      } else {
        v[0] = *reinterpret_cast<const bf16x8_t*>(page[0] + d);
        v[1] = *reinterpret_cast<const bf16x8_t*>(page[1] + d);
      }
      f32x16_t sum = f32x16_t{};
#pragma unroll
      for (int h = 0; h < 2; ++h)
        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kinds_of(v[h]), sees[h], sum, 0, 0, 0);
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int n = (int)sum[x], plus = n & 1023, minus = n >> 10 & 1023;
        const float y = n >> 20 || (plus && minus) ? __builtin_nanf("") : __builtin_inff();
        o[mb][x] += n == 0 ? 0.f : plus ? y : -y;
      }
    }
  }
  if (!row_ok) return;
  const int rows = nt * G, slot_floats = slot_floats_for(rows);
  const Slots sl = group_slots(a.ws, f[DLFP_W_WSGROUP], nsplits, slot_floats);
  const int my = f[DLFP_W_SPLIT] * slot_floats;
  const int64_t orow = ((int64_t)(f[DLFP_W_QROW0] + tr) * a.hq + kh * G + r % G) * D;
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const float y = o[mb][x];
      if (y == 0.f) continue;
      const int chunk = 4 * mb + (x >> 2), dim = 8 * chunk + 4 * hi + (x & 3);
      if (nsplits > 1) {
        const int at = my + (chunk * rows + r) * 8 + 4 * hi + (x & 3);
        pstore1(sl, at, pload1(sl, at) + y);
      } else if (a.out_f32) {
        static_cast<float*>(a.out)[orow + dim] += y;
      } else {
        uint16_t* at = static_cast<uint16_t*>(a.out) + orow + dim;
        const float z = __builtin_bit_cast(float, (uint32_t)*at << 16) + y;
        *at = (uint16_t)pack_bf16(z, z);
      }
    }
}

// ---------------------------------------------------------------- prefill

// Prefill LDS map: K tiles in two slots, V^T tiles in two slots, the unit's block
// ids, and for 8-bit pages their exponent bytes (keys' | values' << 8).
template <bool KV8>
struct PreLds {
  static constexpr int TILE = 4 * page_bytes<KV8>();
  static constexpr int V_BASE = 2 * TILE;
  static constexpr int PTAB = 4 * TILE;
  static constexpr int ETAB = PTAB + 4 * PRE_PTAB;
  static constexpr int BYTES = ETAB + (KV8 ? 2 * PRE_PTAB : 0);
};

// Per wavefront of a decode unit: a key slot and a value slot of one block each
// (32 keys of bf16 pages, 64 of 8-bit ones), ids and exponents of its pages.
constexpr int SLOT = 8192;
template <bool KV8, int NW>
constexpr int decode_wave_lds() {
  return 2 * SLOT + ((DEC_PTAB / NW + 4) * (KV8 ? 6 : 4) + 63) / 64 * 64;
}

template <bool KV8>
constexpr int window_lds() {
  constexpr int pre = PreLds<KV8>::BYTES, dec = 4 * decode_wave_lds<KV8, 1>();
  static_assert(4 * 1024 * 16 + 2 * 4 * 32 * 4 <= (pre > dec ? pre : dec), "four partial results");
  return pre > dec ? pre : dec;
}

// Unit of a tile of 128 query rows (128 / G tokens of G heads): 32 rows a wavefront,
// their keys in tiles of 64 through two slots of LDS that the four share, each key and
// value read from memory once for 128 rows.  32x32 products: the scores of a row are in
// two lanes, so its maximum and sum take one exchange.  Bound by the matrix products
// and the exponentials between them at the clock that their power allows: 4096 tokens
// of 64 heads in a window of 4000 keys, bf16 pages, 538 GFLOP in 495 to 517 us (1.04 to
// 1.09 PFLOP/s; a library product of 8192^3 1.23); 2 x 1999 tokens of 32 heads over
// 8144 keys, 8-bit pages, 457 GFLOP in 392 to 421 us (1.09 to 1.17).  fp32 output has
// three products for one with the values: 1450 tokens of 64 heads over 8533 keys 612 to
// 630 us, with bf16 output 371; of products that is 1.18 to 1.21 PFLOP/s.
template <int G, bool KV8, bool OUT32, bool CAREFUL>
__device__ __forceinline__ void prefill_unit(const Args& a, const record_t f, char* smem,
                                             volatile int* special) {
  using L = PreLds<KV8>;
  constexpr int PB = page_bytes<KV8>();
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int col = lane & 31, hi = lane >> 5;
  const int s = f[DLFP_W_SEQ], kh = f[DLFP_W_KVHEAD];
  const int nt = f[DLFP_W_QNTOK];
  const int vb = f[DLFP_W_KVBEGIN], ve = f[DLFP_W_KVEND];
  const int nsplits = f[DLFP_W_NSPLITS];
  const int row0 = f[DLFP_W_QROW0], pos0 = f[DLFP_W_QPOS0];
  const Span sp = span_of(f);
  const int32_t* bt = a.block_table + (int64_t)s * a.max_blocks;

  const int r = wave * 32 + col;  // this lane's row within the tile
  const int tr = r / G, hh = r % G;
  const bool row_ok = tr < nt;
  // Virtual keys [v_low, v_end) and those below the sinks are this row's; rows past
  // the tile see nothing.
  const int v_end = row_ok ? min(sp.end(pos0 + tr), ve) : 0;
  const int v_low = row_ok ? sp.low(pos0 + tr) : 0;
  const int wave_tok0 = uniform((wave * 32) / G);
  const bool wave_active = wave_tok0 < nt;
  // Keys from wave_end on some row of the wavefront does not see; the position of
  // its last row.
  const int wave_end = min(sp.end(pos0 + wave_tok0), ve);
  const int wave_last = pos0 + min(nt - 1, uniform((wave * 32 + 31) / G));

  // Q^T as the B operand.  Rows past the tile load its first one.
  constexpr bool CODES = KV8 && !OUT32;  // scores from products of codes
  bf16x8_t qf[8];
  {
    const int64_t qrow = ((int64_t)(row0 + (row_ok ? tr : 0)) * a.hq + kh * G + hh) * D;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const int d = KV8 ? 32 * (kk >> 1) + 16 * hi + 8 * (kk & 1) : 16 * kk + 8 * hi;
      qf[kk] = *reinterpret_cast<const bf16x8_t*>(a.q + qrow + d);
    }
  }

  operand8_t q8[2][2];
  int q_exp = 0;
  if constexpr (CODES) q_exp = query_codes(qf, q8);

  const int ntiles = (ve - vb + KV_TILE - 1) / KV_TILE;
  const int first_page = vb / PAGE, npages = (ve - 1) / PAGE - first_page + 1;
  int32_t* ptab = reinterpret_cast<int32_t*>(smem + L::PTAB);
  uint16_t* etab = reinterpret_cast<uint16_t*>(smem + L::ETAB);
  if (!CAREFUL && tid == 0) *special = 0;
#pragma unroll 4
  for (int i = tid; i < npages; i += THREADS) {
    int id = bt[sp.page(first_page + i)];
    if ((unsigned)id >= (unsigned)a.num_blocks) {
      raise_error(a.ws);
      id = 0;
    }
    ptab[i] = id;
  }
  wait_memory_complete();
  __syncthreads();

  // Copies: wave w moves page w of each tile; past the unit's last page, that
  // page again (its keys there are masked).  LDS chunk (16 bytes) x of K row R
  // holds the row's chunk x ^ R (bf16), or x ^ f(R) (8 bits: 8 chunks a row, the
  // rows that LDS serves together are the slots {0-3, 8-11} of two pages).
  constexpr int NC = PB / 1024;  // copies of a page
  uint32_t koff[NC], voff[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int ck = 64 * i + lane;
    if constexpr (KV8) {
      const int rr = ck >> 3;
      koff[i] = rr * 128 + (((ck & 7) ^ ((rr >> 1) & 7) ^ ((wave & 1) << 1)) << 4);
      voff[i] = ck << 4;
    } else {
      const int rr = ck >> 4, d = ck >> 1;
      koff[i] = rr * 256 + (((ck & 15) ^ rr) << 4);
      voff[i] = d * 32 + (((ck & 1) ^ vt_swz(d)) << 4);
    }
  }
  auto page_id = [&](int t) { return ptab[min(4 * t + wave, npages - 1)]; };
  auto page_off = [&](int id) -> int64_t { return ((int64_t)uniform(id) * a.hkv + kh) * PB; };
  const uint32_t lds_wave = lds_addr(smem) + uniform(wave) * PB;
  auto issue_k = [&](int64_t off, int slot) {
    const char* src = uniform_ptr(a.kc + off);
#pragma unroll
    for (int i = 0; i < NC; ++i) lds_copy16(src, koff[i], lds_wave + slot * L::TILE + i * 1024);
  };
  auto issue_v = [&](int64_t off, int slot) {
    const char* src = uniform_ptr(a.vc + off);
#pragma unroll
    for (int i = 0; i < NC; ++i)
      lds_copy16(src, voff[i], lds_wave + L::V_BASE + slot * L::TILE + i * 1024);
  };
  // Values that no row of the unit sees (before the first one's window and no
  // sinks, or past the unit's end) are zeroed in LDS: a probability of 0 times a
  // NaN would still be NaN.  CAREFUL: also those that are not finite, of tiles with
  // keys that not all rows see.  Wavefront w does page w of the tile.
  const int unit_end = CAREFUL ? min(sp.end(pos0), ve) : ve, last = pos0 + (CAREFUL ? nt - 1 : 0);
  auto has_unseen = [&](int t) {
    const int v0 = vb + t * KV_TILE;
    return v0 + KV_TILE > unit_end || sp.below(v0, v0 + KV_TILE, last);
  };
  auto zero_unseen = [&](int slot, int v0) {
    zero_values<KV8, 1, CAREFUL>(smem + L::V_BASE + slot * L::TILE + uniform(wave) * PB, sp,
                                 v0 + uniform(wave) * PAGE, pos0, ve);
  };

  // Per-lane LDS offsets of the operands.
  int kbase, vbase, krow[2];
  if constexpr (KV8) {
    // Row `col` of 32-key block j is position 4 (col / 8) + col % 4 of page
    // 2 j + (col / 4) % 2, so that accumulator register rr of lane half hi is
    // position rr of page 2 j + hi.
    const int pg = (col >> 2) & 1, slot = vt_pos(4 * (col >> 3) + (col & 3));
    kbase = pg * PB + slot * 128;
    krow[0] = ((slot >> 1) & 7) ^ (pg << 1);
    vbase = L::V_BASE + hi * PB + col * 16;
  } else {
    kbase = col * 256 + ((hi ^ (col & 15)) << 4);
    vbase = L::V_BASE + col * 32 + ((hi ^ vt_swz(col)) << 4);
  }

  float m_run = NEG_BIG, l_run = 0.f;
  f32x16_t o[4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) o[mb] = f32x16_t{};
  const float c = a.scale_log2;

  // Scales of a tile's pages: keys' of this lane's row page, values' of page
  // 2 j + hi.
  auto tile_exp = [&](int t, int j, int pg, int shift) {
    return (etab[min(4 * t + 2 * j + pg, npages - 1)] >> shift) & 0xFF;
  };
  auto tile_scale = [&](int t, int j, int pg, int shift) {
    return scale_of(tile_exp(t, j, pg, shift));
  };
  // S^T = K Q^T for the tile in K slot `slot`, two 32-key accumulators.
  auto qk = [&](f32x16_t* sacc, int slot, int t) {
    sacc[0] = f32x16_t{};
    sacc[1] = f32x16_t{};
    if constexpr (CODES) {
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        operand8_t x[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const char* kp = smem + slot * L::TILE + kbase + 2 * j * PB;
          x[j] = operand8(*reinterpret_cast<const codes_t*>(kp + (((4 * d + hi) ^ krow[0]) << 4)),
                          *reinterpret_cast<const codes_t*>(kp + (((4 * d + 2 + hi) ^ krow[0]) << 4)));
        }
#pragma unroll
        for (int term = 0; term < 2; ++term)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            sacc[j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                x[j], q8[term][d], sacc[j], 0, 0, 0, tile_exp(t, j, (col >> 2) & 1, 0), 0,
                q_exp - 4 * term);
      }
    } else if constexpr (KV8) {
      const float s0 = tile_scale(t, 0, (col >> 2) & 1, 0), s1 = tile_scale(t, 1, (col >> 2) & 1, 0);
#pragma unroll
      for (int kk = 0; kk < 8; kk += 2) {
        const char* kp = smem + slot * L::TILE + kbase + (((kk + hi) ^ krow[0]) << 4);
        bf16x8_t x[2], y[2];
        widen(*reinterpret_cast<const codes_t*>(kp), s0, &x[0], &x[1]);
        widen(*reinterpret_cast<const codes_t*>(kp + 2 * PB), s1, &y[0], &y[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          sacc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], qf[kk + i], sacc[0], 0, 0, 0);
          sacc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[i], qf[kk + i], sacc[1], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        const char* kp = smem + slot * L::TILE + (kbase ^ (kk << 5));
        const bf16x8_t k0f = *reinterpret_cast<const bf16x8_t*>(kp);
        const bf16x8_t k1f = *reinterpret_cast<const bf16x8_t*>(kp + 32 * 256);
        sacc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0f, qf[kk], sacc[0], 0, 0, 0);
        sacc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1f, qf[kk], sacc[1], 0, 0, 0);
      }
    }
  };
  // Masks the scores of a tile starting at virtual key v0, where it has to be.
  auto needs_mask = [&](int v0) {
    return v0 + KV_TILE > wave_end || sp.below(v0, v0 + KV_TILE, wave_last);
  };
  auto mask = [&](f32x16_t* sacc, int v0) {
    // Register rr of accumulator j is key v0 + base + at(j, rr).
    const int base = KV8 ? 16 * hi : 4 * hi;
    auto at = [](int j, int rr) {
      return 32 * j + (KV8 ? vt_pos(rr) : 8 * (rr >> 2) + (rr & 3));
    };
    const float none = -__builtin_inff();
    if (v0 + KV_TILE > wave_end) {
      const int n = v_end - v0 - base;
#pragma unroll
      for (int x = 0; x < 32; ++x)
        sacc[x >> 4][x & 15] = at(x >> 4, x & 15) < n ? sacc[x >> 4][x & 15] : none;
    }
    if (sp.below(v0, v0 + KV_TILE, wave_last)) {
      const int n = v_low - v0 - base, m = sp.sinks - v0 - base;
#pragma unroll
      for (int x = 0; x < 32; ++x) {
        const int k = at(x >> 4, x & 15);
        sacc[x >> 4][x & 15] = k >= n || k < m ? sacc[x >> 4][x & 15] : none;
      }
    }
  };
  auto rowmax = [&](const f32x16_t* sacc) {
    float m4[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      m4[i] = fmaxf(sacc[i >> 1][8 * (i & 1)], sacc[i >> 1][8 * (i & 1) + 1]);
#pragma unroll
    for (int rr = 2; rr < 8; ++rr)
#pragma unroll
      for (int i = 0; i < 4; ++i) m4[i] = fmaxf(m4[i], sacc[i >> 1][8 * (i & 1) + rr]);
    return fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
  };
  auto rebase = [&](float mx) {
    const float m_tile = max_xor32(mx) * c;
    if (__builtin_amdgcn_ballot_w64(m_tile > m_run + RESCALE_LOG2)) {
      const float m_new = m_tile > m_run + RESCALE_LOG2 ? m_tile : m_run;
      const float alpha = fexp2(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int mb = 0; mb < 4; ++mb) o[mb] *= alpha;
    }
  };
  // P^T = exp2(S^T c - m) as the B operands of the 16-key steps k0 .. k1 - 1.
  auto probs = [&](f32x16_t* sacc, bf16x8_t* pf, int k0, int k1) {
#pragma unroll
    for (int kk = k0; kk < k1; ++kk) {
      u32x4_t pk;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int x = 8 * (kk & 1) + 2 * w;
        float p0 = fexp2(__builtin_fmaf(sacc[kk >> 1][x], c, -m_run));
        float p1 = fexp2(__builtin_fmaf(sacc[kk >> 1][x + 1], c, -m_run));
        if constexpr (OUT32) {
          l_run += p0 + p1;
          pk[w] = cut(p0, p1);
          sacc[kk >> 1][x] = p0;
          sacc[kk >> 1][x + 1] = p1;
        } else {
          pk[w] = pack_bf16(p0, p1);
        }
      }
      pf[kk] = __builtin_bit_cast(bf16x8_t, pk);
    }
  };
  // The next term of the probabilities (fp32 output): what the terms before left.
  auto next_term = [&](f32x16_t* sacc, bf16x8_t* pf, bool last) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      u32x4_t pk = __builtin_bit_cast(u32x4_t, pf[kk]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int x = 8 * (kk & 1) + 2 * w;
        float p0 = sacc[kk >> 1][x], p1 = sacc[kk >> 1][x + 1];
        pk[w] = above_zero<KV8>(last ? pack_bf16(p0, p1) : cut(p0, p1), pk[w]);
        sacc[kk >> 1][x] = p0;
        sacc[kk >> 1][x + 1] = p1;
      }
      pf[kk] = __builtin_bit_cast(bf16x8_t, pk);
    }
  };
  // Row sum of the rounded probabilities (this half of the row).
  auto rowsum = [&](const bf16x8_t* pf) {
    if constexpr (OUT32) return;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const u32x4_t pk = __builtin_bit_cast(u32x4_t, pf[kk]);
#pragma unroll
      for (int w = 0; w < 4; ++w) l_run = dot2(pk[w], 0x3F803F80u, l_run);  // two bf16 1.0
    }
  };
  // O^T += V^T P^T over the 32-key halves j0 .. j1 - 1 of the tile in V slot `slot`.
  auto pv = [&](const bf16x8_t* pf, int slot, int t, int j0, int j1) {
#pragma unroll
    for (int j = j0; j < j1; ++j) {
      if constexpr (KV8) {
        const float vs = tile_scale(t, j, hi, 8);
#pragma unroll
        for (int mb = 0; mb < 4; ++mb) {
          bf16x8_t vf[2];
          widen(*reinterpret_cast<const codes_t*>(smem + vbase + slot * L::TILE + 2 * j * PB + mb * 512),
                vs, &vf[0], &vf[1]);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], pf[2 * j + i], o[mb], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int kk = 2 * j; kk < 2 * j + 2; ++kk)
#pragma unroll
          for (int mb = 0; mb < 4; ++mb) {
            const bf16x8_t vf = *reinterpret_cast<const bf16x8_t*>(smem + vbase + slot * L::TILE +
                                                                   kk * PB + mb * 1024);
            o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[kk], o[mb], 0, 0, 0);
          }
      }
    }
  };

  // Tiles 0 (K and V) and 1 (K) in flight, then S_0.
  int64_t off_next = page_off(page_id(0));
  issue_k(off_next, 0);
  issue_v(off_next, 0);
  if (ntiles > 1) {
    off_next = page_off(page_id(1));
    issue_k(off_next, 1);
  }
  if constexpr (KV8) {  // with the first tiles on their way
#pragma unroll 4
    for (int i = tid; i < npages; i += THREADS) {
      const int64_t e = (int64_t)ptab[i] * a.hkv + kh;
      etab[i] = (uint16_t)(a.k_exp[e] | a.v_exp[e] << 8);
    }
  }
  wait_memory_complete();
  __syncthreads();
  if (has_unseen(0)) {
    zero_unseen(0, vb);
    __syncthreads();
  }
  f32x16_t sa[2], sb[2];
  if (wave_active) {
    qk(sa, 0, 0);
    if (needs_mask(vb)) mask(sa, vb);
    rebase(rowmax(sa));
  }
  __syncthreads();  // K slot 0 is refilled below
  int id2 = page_id(2);  // read a step before its use

  // Step j: loads of K_{j+2} and V_{j+1} go out; S_{j+1} = K_{j+1} Q^T beside the
  // first half of tile j's exponentials; the second half beside the first half of
  // O += V_j P_j; the row maxima of tile j + 1 beside the rest.
  auto step = [&](int j, f32x16_t* cur, f32x16_t* nxt, auto parity) {
    constexpr int PAR = decltype(parity)::value;  // j & 1
    const bool more = j + 1 < ntiles;
    if (more) issue_v(off_next, PAR ^ 1);
    if (j + 2 < ntiles) {
      off_next = page_off(id2);
      issue_k(off_next, PAR);
    }
    id2 = page_id(j + 3);
    if (wave_active) {
      bf16x8_t pf[4];
      // On the last tile this reads a stale slot; the result is not used.  With
      // fp32 output the probabilities stay in registers for their three terms, and
      // the next scores come after them.
      if constexpr (!OUT32) qk(nxt, PAR ^ 1, j + 1);
      probs(cur, pf, 0, 2);
      if constexpr (!KV8 && !OUT32) {
        // Key operands four products ahead, exponentials between the products.
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      }
      __builtin_amdgcn_s_setprio(1);
      probs(cur, pf, 2, 4);
      pv(pf, PAR, j, 0, 1);
      if constexpr (!KV8 && !OUT32) {
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
          __builtin_amdgcn_sched_group_barrier(0x002, 5, 1);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      pv(pf, PAR, j, 1, 2);
      rowsum(pf);
      if constexpr (OUT32) {
        next_term(cur, pf, false);
        pv(pf, PAR, j, 0, 2);
        next_term(cur, pf, true);
        pv(pf, PAR, j, 0, 2);
        qk(nxt, PAR ^ 1, j + 1);
      }
      float mx = rowmax(nxt);
      if constexpr (!KV8 && !OUT32) {
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 2);
          __builtin_amdgcn_sched_group_barrier(0x002, 5, 2);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 2);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      if (more) {
        const int v1 = vb + (j + 1) * KV_TILE;
        if (needs_mask(v1)) {
          mask(nxt, v1);
          mx = rowmax(nxt);
        }
        rebase(mx);
      }
    }
    wait_memory_complete();
    __syncthreads();
    if (more && has_unseen(j + 1)) {
      zero_unseen(PAR ^ 1, vb + (j + 1) * KV_TILE);
      __syncthreads();
    }
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  for (int j = 0; j < ntiles; j += 2) {
    step(j, sa, sb, even);
    if (j + 1 < ntiles) step(j + 1, sb, sa, odd);
  }

  if (!CAREFUL && row_ok && !all_finite(o)) *special = 1;
  l_run = sum_xor32(l_run);
  const int rows = nt * G;
  // o[mb][rr] = O[row][32 mb + 8 (rr / 4) + 4 hi + rr % 4]
  if (nsplits == 1) {
    // Through the wavefront's part of the tiles' LDS, so that stores are whole
    // rows: a row's 16-byte chunk x sits at x ^ row.
    if (!wave_active) return;
    constexpr int ROW = OUT32 ? 512 : 256, CHUNKS = ROW / 16;
    static_assert(128 * ROW <= window_lds<KV8>(), "the tile's rows");
    char* rows_lds = smem + wave * 32 * ROW;
    const float inv = 1.f / l_run;
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = o[mb][4 * g4 + i] * inv;
        char* row = rows_lds + col * ROW;
        if constexpr (OUT32)
          *reinterpret_cast<f32x4_t*>(row + (((8 * mb + 2 * g4 + hi) ^ col) << 4)) =
              f32x4_t{x[0], x[1], x[2], x[3]};
        else
          *reinterpret_cast<u32x2_t*>(row + (((4 * mb + g4) ^ (col & 15)) << 4) + 8 * hi) =
              u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
      }
    wave_sync();
    char* out = static_cast<char*>(a.out);
#pragma unroll
    for (int i = 0; i < 32 * CHUNKS / 64; ++i) {
      const int at = 64 * i + lane, lr = at / CHUNKS, x = at % CHUNKS;
      const int rr = wave * 32 + lr, t = rr / G;
      const u32x4_t v =
          *reinterpret_cast<const u32x4_t*>(rows_lds + lr * ROW + ((x ^ (lr & (CHUNKS - 1))) << 4));
      if (t < nt)
        *reinterpret_cast<u32x4_t*>(
            out + ((int64_t)(row0 + t) * a.hq + kh * G + rr % G) * ROW + 16 * x) = v;
    }
    return;
  }

  // Partial result, in the layout that prefill_merge reads.
  const int slot_floats = slot_floats_for(rows);
  const Slots sl = group_slots(a.ws, f[DLFP_W_WSGROUP], nsplits, slot_floats);
  const int my = f[DLFP_W_SPLIT] * slot_floats;
  if (row_ok) {
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const f32x4_t v = {o[mb][4 * g4], o[mb][4 * g4 + 1], o[mb][4 * g4 + 2],
                           o[mb][4 * g4 + 3]};
        pstore4(sl, my + ((4 * mb + g4) * rows + r) * 8 + 4 * hi, v);
      }
    if (hi == 0) {
      pstore1(sl, my + rows * D + r, m_run);
      pstore1(sl, my + rows * D + rows + r, l_run);
    }
  }
}

// Keys of a block of a unit of few rows.
template <bool KV8>
constexpr int SMALL_KEYS = SLOT / page_bytes<KV8>() * PAGE;

// Unit of at most 32 query rows: one wavefront holds all of them, so the four
// split the keys instead: wavefront w takes blocks w, w + 4, ... of the unit, each
// through a key slot and a value slot of its own, without a barrier until the
// four results are added through LDS.  Block and slots as a decode unit's (32 keys
// of bf16 pages, 64 of 8-bit ones), products, masks and layouts as a tile's.  Bound by
// a wavefront's chain of steps: a quarter of the keys each, where a tile of as many
// rows has one wavefront for all.  64 tokens of 16 heads over 264 keys 8.7 us, as a
// tile 12.2; 256 over 1256 15.4 and 20.1; 2048 over 4048, where the rows fill the
// chip, 86 and 68, each key being read four times as often.
template <int G, bool KV8, bool OUT32, bool CAREFUL>
__device__ __forceinline__ void small_unit(const Args& a, const record_t f, char* smem,
                                           volatile int* special) {
  constexpr int PB = page_bytes<KV8>();
  constexpr int BP = SLOT / PB;     // pages of a block
  constexpr int KEYS = SMALL_KEYS<KV8>;
  constexpr int NJ = BP / 2;        // 32-key products of a block
  constexpr int NC = PB / 1024;     // copies of a page
  constexpr bool CODES = KV8 && !OUT32;
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const int col = lane & 31, hi = lane >> 5;
  char* wl = smem + wave * decode_wave_lds<KV8, 4>();
  const int s = f[DLFP_W_SEQ], kh = f[DLFP_W_KVHEAD], nt = f[DLFP_W_QNTOK];
  const int vb = f[DLFP_W_KVBEGIN], ve = f[DLFP_W_KVEND];
  const int nsplits = f[DLFP_W_NSPLITS];
  const int row0 = f[DLFP_W_QROW0], pos0 = f[DLFP_W_QPOS0];
  const Span sp = span_of(f);
  const int32_t* bt = a.block_table + (int64_t)s * a.max_blocks;
  int32_t* ptab = reinterpret_cast<int32_t*>(wl + 2 * SLOT);
  uint16_t* etab = reinterpret_cast<uint16_t*>(ptab + DEC_PTAB / 4 + 4);

  const int tr = col / G, hh = col % G;
  const bool row_ok = tr < nt;
  const int v_end = row_ok ? min(sp.end(pos0 + tr), ve) : 0;
  const int v_low = row_ok ? sp.low(pos0 + tr) : 0;
  const int unit_end = min(sp.end(pos0), ve), last = pos0 + nt - 1;

  const int first_page = vb / PAGE;
  const int npages = (ve + PAGE - 1) / PAGE - first_page, nblocks = (npages + BP - 1) / BP;
  const int mine = nblocks > wave ? (nblocks - wave + 3) / 4 : 0;
  auto page_of = [&](int i, int h) { return min(BP * (wave + 4 * i) + h, npages - 1); };
  auto pages_in = [&](int i) { return min(BP, npages - BP * (wave + 4 * i)); };
  for (int x = lane; x < BP * mine; x += 64) {
    int id = bt[sp.page(first_page + page_of(x / BP, x % BP))];
    if ((unsigned)id >= (unsigned)a.num_blocks) {
      raise_error(a.ws);
      id = 0;
    }
    ptab[x] = id;
  }
  bf16x8_t qf[8];
  {
    const int64_t qrow = ((int64_t)(row0 + (row_ok ? tr : 0)) * a.hq + kh * G + hh) * D;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const int d = KV8 ? 32 * (kk >> 1) + 16 * hi + 8 * (kk & 1) : 16 * kk + 8 * hi;
      qf[kk] = *reinterpret_cast<const bf16x8_t*>(a.q + qrow + d);
    }
  }
  wait_memory_complete();
  wave_sync();

  uint32_t kofs[NC], vofs[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int ck = 64 * j + lane;
    if constexpr (KV8) {
      const int R = ck >> 3;
      kofs[j] = R * 128 + (((ck & 7) ^ ((R >> 1) & 7)) << 4);
      vofs[j] = ck << 4;
    } else {
      const int R = ck >> 4, d = ck >> 1;
      kofs[j] = R * 256 + (((ck & 15) ^ R) << 4);
      vofs[j] = d * 32 + (((ck & 1) ^ vt_swz(d)) << 4);
    }
  }
  const uint32_t lds_wave = (uint32_t)uniform((int)lds_addr(wl));
  auto issue_k = [&](int i) {
    const int n = pages_in(i);
#pragma unroll
    for (int h = 0; h < BP; ++h) {
      if (h >= n) break;
      const char* src = a.kc + ((int64_t)uniform(ptab[BP * i + h]) * a.hkv + kh) * PB;
      const uint32_t x = KV8 ? (h & 1) << 5 : 0;
#pragma unroll
      for (int j = 0; j < NC; ++j) lds_copy16(src + (kofs[j] ^ x), lds_wave + h * PB + j * 1024);
    }
  };
  auto issue_v = [&](int i) {
    const int n = pages_in(i);
#pragma unroll
    for (int h = 0; h < BP; ++h) {
      if (h >= n) break;
      const char* src = a.vc + ((int64_t)uniform(ptab[BP * i + h]) * a.hkv + kh) * PB;
#pragma unroll
      for (int j = 0; j < NC; ++j) lds_copy16(src + vofs[j], lds_wave + SLOT + h * PB + j * 1024);
    }
  };
  if (mine > 0) {
    issue_k(0);
    issue_v(0);
  }
  if constexpr (KV8) {
    for (int x = lane; x < BP * mine; x += 64) {
      const int64_t e = (int64_t)ptab[x] * a.hkv + kh;
      etab[x] = (uint16_t)(a.k_exp[e] | a.v_exp[e] << 8);
    }
    wave_sync();
  }
  operand8_t q8[2][2];
  int q_exp = 0;
  if constexpr (CODES) q_exp = query_codes(qf, q8);

  // Operand offsets, as in prefill_unit.
  int kbase, vbase, kxor = 0;
  const int kpg = (col >> 2) & 1;
  if constexpr (KV8) {
    const int slot = vt_pos(4 * (col >> 3) + (col & 3));
    kbase = kpg * PB + slot * 128;
    kxor = ((slot >> 1) & 7) ^ (kpg << 1);
    vbase = SLOT + hi * PB + col * 16;
  } else {
    kbase = col * 256 + ((hi ^ (col & 15)) << 4);
    vbase = SLOT + col * 32 + ((hi ^ vt_swz(col)) << 4);
  }
  float m_run = NEG_BIG, l_run = 0.f;
  f32x16_t o[4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) o[mb] = f32x16_t{};
  const float c = a.scale_log2;
  if (!CAREFUL && tid == 0) *special = 0;

  for (int i = 0; i < mine; ++i) {
    const int v0 = vb + KEYS * (wave + 4 * i);
    const bool more = i + 1 < mine;
    if (pages_in(i) == BP)
      wait_copies<8>();  // in flight, oldest first: this block's keys, its values
    else
      wait_copies<0>();
    f32x16_t sacc[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) sacc[j] = f32x16_t{};
    if constexpr (CODES) {
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const char* kp = wl + kbase + 2 * j * PB;
          const operand8_t x = operand8(
              *reinterpret_cast<const codes_t*>(kp + (((4 * d + hi) ^ kxor) << 4)),
              *reinterpret_cast<const codes_t*>(kp + (((4 * d + 2 + hi) ^ kxor) << 4)));
          const int ke = etab[BP * i + 2 * j + kpg] & 0xFF;
#pragma unroll
          for (int term = 0; term < 2; ++term)
            sacc[j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                x, q8[term][d], sacc[j], 0, 0, 0, ke, 0, q_exp - 4 * term);
        }
    } else if constexpr (KV8) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const float ks = scale_of(etab[BP * i + 2 * j + kpg] & 0xFF);
#pragma unroll
        for (int kk = 0; kk < 8; kk += 2) {
          bf16x8_t x[2];
          widen(*reinterpret_cast<const codes_t*>(wl + kbase + 2 * j * PB + (((kk + hi) ^ kxor) << 4)),
                ks, &x[0], &x[1]);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            sacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[h], qf[kk + h], sacc[j], 0, 0, 0);
        }
      }
    } else {
      bf16x8_t kf[8];
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        kf[kk] = *reinterpret_cast<const bf16x8_t*>(wl + (kbase ^ (kk << 5)));
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        sacc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[kk], sacc[0], 0, 0, 0);
    }
    wait_lds();  // the key slot is free
    if (more) issue_k(i + 1);
    const bool next_full = more && pages_in(i + 1) == BP;
    // Masks, as in prefill_unit.
    const int base = KV8 ? 16 * hi : 4 * hi;
    auto at = [](int x) {
      return 32 * (x >> 4) + (KV8 ? vt_pos(x & 15) : 8 * ((x & 15) >> 2) + (x & 3));
    };
    if (v0 + KEYS > unit_end) {
      const int n = v_end - v0 - base;
#pragma unroll
      for (int x = 0; x < 16 * NJ; ++x)
        sacc[x >> 4][x & 15] = at(x) < n ? sacc[x >> 4][x & 15] : -__builtin_inff();
    }
    if (sp.below(v0, v0 + KEYS, last)) {
      const int n = v_low - v0 - base, m = sp.sinks - v0 - base;
#pragma unroll
      for (int x = 0; x < 16 * NJ; ++x)
        sacc[x >> 4][x & 15] = at(x) >= n || at(x) < m ? sacc[x >> 4][x & 15] : -__builtin_inff();
    }
    float mx = -__builtin_inff();
#pragma unroll
    for (int x = 0; x < 16 * NJ; ++x) mx = fmaxf(mx, sacc[x >> 4][x & 15]);
    const float m_tile = max_xor32(mx) * c;
    if (__builtin_amdgcn_ballot_w64(m_tile > m_run + RESCALE_LOG2)) {
      const float m_new = m_tile > m_run + RESCALE_LOG2 ? m_tile : m_run;
      const float alpha = fexp2(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int mb = 0; mb < 4; ++mb) o[mb] *= alpha;
    }
    bf16x8_t pf[2 * NJ];
#pragma unroll
    for (int kk = 0; kk < 2 * NJ; ++kk) {
      u32x4_t pk;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int x = 8 * (kk & 1) + 2 * w;
        float p0 = fexp2(__builtin_fmaf(sacc[kk >> 1][x], c, -m_run));
        float p1 = fexp2(__builtin_fmaf(sacc[kk >> 1][x + 1], c, -m_run));
        if constexpr (OUT32) {
          l_run += p0 + p1;
          pk[w] = cut(p0, p1);
          sacc[kk >> 1][x] = p0;
          sacc[kk >> 1][x + 1] = p1;
        } else {
          pk[w] = pack_bf16(p0, p1);
          l_run = dot2(pk[w], 0x3F803F80u, l_run);  // two bf16 1.0
        }
      }
      pf[kk] = __builtin_bit_cast(bf16x8_t, pk);
    }
    if (next_full)
      wait_copies<8>();  // the values; behind them the next block's keys
    else
      wait_copies<0>();
    if (CAREFUL ? v0 + KEYS > unit_end || sp.below(v0, v0 + KEYS, last)
                : v0 + KEYS > ve || sp.below(v0, v0 + KEYS, pos0)) {
      zero_values<KV8, BP, CAREFUL>(wl + SLOT, sp, v0, pos0, ve);
      wave_sync();
    }
    auto pv = [&]() {
#pragma unroll
      for (int kk = 0; kk < 2 * NJ; kk += KV8 ? 2 : 1)
#pragma unroll
        for (int mb = 0; mb < 4; ++mb) {
          if constexpr (KV8) {
            bf16x8_t x[2];
            widen(*reinterpret_cast<const codes_t*>(wl + vbase + kk * PB + mb * 512),
                  scale_of(etab[BP * i + kk + hi] >> 8), &x[0], &x[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
              o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[h], pf[kk + h], o[mb], 0, 0, 0);
          } else {
            const bf16x8_t vf =
                *reinterpret_cast<const bf16x8_t*>(wl + vbase + kk * PB + mb * 1024);
            o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[kk], o[mb], 0, 0, 0);
          }
        }
    };
    pv();
    if constexpr (OUT32) {
#pragma unroll
      for (int term = 0; term < 2; ++term) {
#pragma unroll
        for (int kk = 0; kk < 2 * NJ; ++kk) {
          u32x4_t pk = __builtin_bit_cast(u32x4_t, pf[kk]);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int x = 8 * (kk & 1) + 2 * w;
            float p0 = sacc[kk >> 1][x], p1 = sacc[kk >> 1][x + 1];
            pk[w] = above_zero<KV8>(term ? pack_bf16(p0, p1) : cut(p0, p1), pk[w]);
            sacc[kk >> 1][x] = p0;
            sacc[kk >> 1][x + 1] = p1;
          }
          pf[kk] = __builtin_bit_cast(bf16x8_t, pk);
        }
        pv();
      }
    }
    wait_lds();  // the value slot is free
    if (more) issue_v(i + 1);
  }

  // Add the four wavefronts' results through LDS.  Piece (chunk, hi) of a row holds
  // dims 32 (chunk / 4) + 8 (chunk % 4) + 4 hi .. + 3; thread (row, sub) takes chunks
  // 2 sub and 2 sub + 1, 16 consecutive dims; the row is XORed with the chunk so that
  // both sides spread over the banks.
  l_run = sum_xor32(l_run);
  wait_memory_complete();
  __syncthreads();  // every wavefront is done with its slots
  if (!CAREFUL && row_ok && !all_finite(o)) *special = 1;
  f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);
  float* stat = reinterpret_cast<float*>(smem + 4 * 1024 * 16);  // m[4][32], l[4][32]
  auto at = [](int w, int ch, int h, int row) {
    return w * 1024 + ch * 64 + h * 32 + (row ^ (((ch >> 1) & 7) << 1));
  };
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      red[at(wave, 4 * mb + g4, hi, col)] = f32x4_t{o[mb][4 * g4], o[mb][4 * g4 + 1],
                                                   o[mb][4 * g4 + 2], o[mb][4 * g4 + 3]};
  if (hi == 0) {
    stat[wave * 32 + col] = m_run;
    stat[128 + wave * 32 + col] = l_run;
  }
  __syncthreads();
  const int row = tid >> 3, sub = tid & 7, rows = nt * G;
  float M = NEG_BIG, L = 0.f, wgt[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, stat[w * 32 + row]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    wgt[w] = fexp2(stat[w * 32 + row] - M);
    L += wgt[w] * stat[128 + w * 32 + row];
  }
  f32x4_t acc[4];  // pieces (2 sub, 0), (2 sub, 1), (2 sub + 1, 0), (2 sub + 1, 1)
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    acc[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) acc[x] += wgt[w] * red[at(w, 2 * sub + (x >> 1), x & 1, row)];
  }
  if (nsplits == 1) {
    if (row < rows) {
      const float inv = 1.f / L;
      const int64_t orow = ((int64_t)(row0 + row / G) * a.hq + kh * G + row % G) * D + 16 * sub;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        store4(a, orow + 4 * x, acc[x][0] * inv, acc[x][1] * inv, acc[x][2] * inv, acc[x][3] * inv);
    }
    return;
  }
  const int slot_floats = slot_floats_for(rows);
  const Slots sl = group_slots(a.ws, f[DLFP_W_WSGROUP], nsplits, slot_floats);
  const int my = f[DLFP_W_SPLIT] * slot_floats;
  if (row < rows) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      pstore4(sl, my + ((2 * sub + (x >> 1)) * rows + row) * 8 + 4 * (x & 1), acc[x]);
    if (sub == 0) {
      pstore1(sl, my + rows * D + row, M);
      pstore1(sl, my + rows * D + rows + row, L);
    }
  }
}

// A prompt's unit: its rows, stored as results or as partial ones, and, by the
// unit of a split group that comes so far last, the merge.
template <int G, bool KV8, bool OUT32>
__device__ __forceinline__ void prompt_unit(const Args& a, const record_t f, char* smem, int* flag,
                                            volatile int* special) {
  const int tid = threadIdx.x, wave = uniform(tid >> 6);
  const int rows = f[DLFP_W_QNTOK] * G, nsplits = f[DLFP_W_NSPLITS];
  if (rows <= SMALL_ROWS)
    small_unit<G, KV8, OUT32, false>(a, f, smem, special);
  else
    prefill_unit<G, KV8, OUT32, false>(a, f, smem, special);
  __syncthreads();
  if (uniform(*special)) {
    if (rows <= SMALL_ROWS)
      small_unit<G, KV8, OUT32, true>(a, f, smem, special);
    else
      prefill_unit<G, KV8, OUT32, true>(a, f, smem, special);
    wait_memory_complete();  // the rows that it adds to
    __syncthreads();
    if (32 * wave < rows)
      add_special<G, KV8>(a, f, 32 * wave, rows <= SMALL_ROWS ? SMALL_KEYS<KV8> : KV_TILE);
  }
  if (nsplits == 1) return;
  wait_memory_complete();
  __syncthreads();  // every wave of the unit has completed its stores
  const int grp = f[DLFP_W_GROUP], slot_floats = slot_floats_for(rows);
  if (tid == 0) *flag = arrive(a.ws, grp) == nsplits - 1;
  __syncthreads();
  if (!*flag) return;
  const Slots sl = group_slots(a.ws, f[DLFP_W_WSGROUP], nsplits, slot_floats);
  const int row0 = f[DLFP_W_QROW0], kh = f[DLFP_W_KVHEAD];
  if (rows > 64)
    prefill_merge<G, 2, Args, true>(a, sl, slot_floats, nsplits, rows, row0, kh);
  else if (rows > 32)
    prefill_merge<G, 4, Args, true>(a, sl, slot_floats, nsplits, rows, row0, kh);
  else
    prefill_merge<G, 8, Args, true>(a, sl, slot_floats, nsplits, rows, row0, kh);
  if (tid == 0)
    __hip_atomic_store(group_counter(a.ws, grp), 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---------------------------------------------------------------- decode

// Decode unit of NW wavefronts: wavefront w takes blocks w, w + NW, ... of the unit;
// their results meet in LDS, those of split ranges in memory.  NW 1: the wavefront
// has no others to wait for, whatever the workgroup.
// The unit's g heads are columns 0-7 of 16x16 products and, with the second term
// of the probabilities, columns 8-15.  Lane l owns column l % 16; its group
// q = l / 16 owns, of 8-bit pages, the 16 keys of page q of the block, of bf16
// pages the eight at positions 8 (q / 2) .. of page q % 2.  Every key and value is
// read once, straight to LDS, for its g heads, and bounds the unit: 256 decoders of a
// 4096-key window, bf16 pages, 4.24 GB in 665 us (6.4 TB/s), 128 of 1024 to 8192 keys,
// 8-bit pages, 1.21 GB in 194 us (6.2 TB/s).
template <int G, bool KV8, bool OUT32, int NW>
__device__ __forceinline__ void decode_unit(const Args& a, const int32_t* rec, char* smem, int* flag) {
  static_assert(G >= 1 && G <= 8, "heads");
  constexpr int PB = page_bytes<KV8>();
  constexpr int BP = SLOT / PB;       // pages of a block
  constexpr int NCH = KV8 ? 4 : 2;    // 16-key products of a block
  constexpr int NC = PB / 1024;       // copies of a page
  constexpr bool CODES = KV8 && !OUT32;
  const int tid = NW == 1 ? threadIdx.x & 63 : threadIdx.x, wave = uniform(tid >> 6);
  const int lane = tid & 63;
  auto meet = [] {
    if constexpr (NW == 1)
      wave_sync();
    else
      __syncthreads();
  };
  char* wl = smem + wave * decode_wave_lds<KV8, NW>();
  const int col = lane & 15, gq = lane >> 4, head = col & 7;
  const record_t f = load_record(rec);
  const int s = f[DLFP_W_SEQ], kh = f[DLFP_W_KVHEAD];
  const int vb = f[DLFP_W_KVBEGIN], ve = f[DLFP_W_KVEND];
  const int nsplits = f[DLFP_W_NSPLITS];
  const int tok = f[DLFP_W_QROW0], pos = f[DLFP_W_QPOS0];
  const Span sp = span_of(f);
  const int32_t* bt = a.block_table + (int64_t)s * a.max_blocks;
  int32_t* ptab = reinterpret_cast<int32_t*>(wl + 2 * SLOT);
  uint16_t* etab = reinterpret_cast<uint16_t*>(ptab + DEC_PTAB / NW + 4);

  const int first_page = vb / PAGE;
  const int npages = (ve + PAGE - 1) / PAGE - first_page, nblocks = (npages + BP - 1) / BP;
  const int mine = nblocks > wave ? (nblocks - wave + NW - 1) / NW : 0;
  // Page h of this wavefront's block i (past the unit's last page, that page);
  // pages that the block has.
  auto page_of = [&](int i, int h) { return min(BP * (wave + NW * i) + h, npages - 1); };
  auto pages_in = [&](int i) { return min(BP, npages - BP * (wave + NW * i)); };

  // Ids of the wavefront's pages; the queries as the B operand.
  for (int x = lane; x < BP * mine; x += 64) {
    int id = bt[sp.page(first_page + page_of(x / BP, x % BP))];
    if ((unsigned)id >= (unsigned)a.num_blocks) {
      raise_error(a.ws);
      id = 0;
    }
    ptab[x] = id;
  }
  bf16x8_t qb[4];
  {
    const uint16_t* qp = a.q + ((int64_t)tok * a.hq + kh * G + min(head, G - 1)) * D;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const int d = KV8 ? 64 * (kk >> 1) + 16 * gq + 8 * (kk & 1) : 32 * kk + 8 * gq;
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(qp + d);
      qb[kk] = __builtin_bit_cast(bf16x8_t, head < G ? v : u32x4_t{0u, 0u, 0u, 0u});
    }
  }
  operand8_t q8;
  int q_exp = 0;
  if constexpr (CODES) {  // the high terms in columns 0-7, the low ones in 8-15
    float m = 0.f;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) m = fmaxf(m, largest(qb[kk]));
    const int e = row_exponent(max_xor32(max_xor16(m)));
    q_exp = col >= 8 ? e - 4 : e;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint32_t hw[2], lw[2];
      split_codes(qb[kk], e, hw, lw);
#pragma unroll
      for (int w = 0; w < 2; ++w) q8[2 * kk + w] = (int)(col >= 8 ? lw[w] : hw[w]);
    }
  }
  wait_memory_complete();
  wave_sync();

  // Copies.  LDS chunk x of K row R of page h holds the row's chunk x ^ R ^ 8 h
  // (bf16), x ^ (R / 2 % 2) ^ 2 h (8 bits); V^T rows of bf16 pages (32 bytes) keep
  // their halves swapped when vt_swz(d), those of 8-bit pages are as stored.
  uint32_t kofs[NC], vofs[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int ck = 64 * j + lane;
    if constexpr (KV8) {
      const int R = ck >> 3;
      kofs[j] = R * 128 + (((ck & 7) ^ ((R >> 1) & 1)) << 4);
      vofs[j] = ck << 4;
    } else {
      const int R = ck >> 4, d = ck >> 1;
      kofs[j] = R * 256 + (((ck & 15) ^ R) << 4);
      vofs[j] = d * 32 + (((ck & 1) ^ vt_swz(d)) << 4);
    }
  }
  const uint32_t lds_wave = (uint32_t)uniform((int)lds_addr(wl));
  auto issue_k = [&](int i) {
    const int n = pages_in(i);
#pragma unroll
    for (int h = 0; h < BP; ++h) {
      if (h >= n) break;
      const char* src = a.kc + ((int64_t)uniform(ptab[BP * i + h]) * a.hkv + kh) * PB;
      const uint32_t x = KV8 ? h << 5 : h << 7;
#pragma unroll
      for (int j = 0; j < NC; ++j) lds_copy16_nt(src + (kofs[j] ^ x), lds_wave + h * PB + j * 1024);
    }
  };
  auto issue_v = [&](int i) {
    const int n = pages_in(i);
#pragma unroll
    for (int h = 0; h < BP; ++h) {
      if (h >= n) break;
      const char* src = a.vc + ((int64_t)uniform(ptab[BP * i + h]) * a.hkv + kh) * PB;
#pragma unroll
      for (int j = 0; j < NC; ++j)
        lds_copy16_nt(src + vofs[j], lds_wave + SLOT + h * PB + j * 1024);
    }
  };
  if (mine > 0) {
    issue_k(0);
    issue_v(0);
  }
  if constexpr (KV8) {  // with the first block on its way
    for (int x = lane; x < BP * mine; x += 64) {
      const int64_t e = (int64_t)ptab[x] * a.hkv + kh;
      etab[x] = (uint16_t)(a.k_exp[e] | a.v_exp[e] << 8);
    }
    wave_sync();
  }

  float m_run = NEG_BIG, l_run = 0.f;
  f32x4_t o[8];
#pragma unroll
  for (int mb = 0; mb < 8; ++mb) o[mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const float c = a.scale_log2;
  // Rows of the K operand: 8 bits, product b: row r is position 4 b + r % 4 of
  // page r / 4; bf16: position 8 (r / 8) + 4 b + r % 4 of page r / 4 % 2.  Rows
  // 4 q .. of the accumulators are then the keys of lane group q.
  const int kpage = KV8 ? col >> 2 : (col >> 2) & 1;
  int krow[NCH], kxor[NCH];
#pragma unroll
  for (int b = 0; b < NCH; ++b) {
    const int R = vt_pos(KV8 ? 4 * b + (col & 3) : 8 * (col >> 3) + 4 * b + (col & 3));
    krow[b] = kpage * PB + R * (KV8 ? 128 : 256);
    kxor[b] = KV8 ? ((R >> 1) & 1) ^ (kpage << 1) : R ^ (kpage << 3);
  }
  const int vpage = KV8 ? gq : gq & 1;  // page of this lane group's keys
  // Slot of its first key of product b.
  auto slot_of = [&](int b) { return vt_pos(KV8 ? 4 * b : 8 * (gq >> 1) + 4 * b); };
  const int vbyte = SLOT + vpage * PB + (KV8 ? col * 16 : col * 32 + (((gq >> 1) ^ vt_swz(col)) << 4));

  for (int i = 0; i < mine; ++i) {
    const int v0 = vb + BP * PAGE * (wave + NW * i);  // first virtual key of the block
    const int n = pages_in(i);
    const bool more = i + 1 < mine, full = n == BP;
    const bool edge = v0 + BP * PAGE > ve || sp.below(v0, v0 + BP * PAGE, pos);
    // In flight, oldest first: this block's keys, its values (eight copies each
    // of a full block; others are the unit's last).
    if (full)
      wait_copies<8>();
    else
      wait_copies<0>();
    float sc[4 * NCH];
    {
      f32x4_t sacc[NCH];
#pragma unroll
      for (int b = 0; b < NCH; ++b) sacc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if constexpr (KV8) {
        const int ke = etab[BP * i + kpage] & 0xFF;
        const float ks = scale_of(ke);
        codes_t kc[NCH][2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int b = 0; b < NCH; ++b)
            kc[b][j] = *reinterpret_cast<const codes_t*>(wl + krow[b] + (((4 * j + gq) ^ kxor[b]) << 4));
        if constexpr (CODES) {
#pragma unroll
          for (int b = 0; b < NCH; ++b)
            sacc[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                operand8(kc[b][0], kc[b][1]), q8, sacc[b], 0, 0, 0, ke, 0, q_exp);
        } else
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int b = 0; b < NCH; ++b) {
            bf16x8_t x[2];
            widen(kc[b][j], ks, &x[0], &x[1]);
            sacc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[0], qb[2 * j], sacc[b], 0, 0, 0);
            sacc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[1], qb[2 * j + 1], sacc[b], 0, 0, 0);
          }
      } else {
        bf16x8_t kf[NCH][4];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int b = 0; b < NCH; ++b)
            kf[b][kk] =
                *reinterpret_cast<const bf16x8_t*>(wl + krow[b] + (((4 * kk + gq) ^ kxor[b]) << 4));
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int b = 0; b < NCH; ++b)
            sacc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[b][kk], qb[kk], sacc[b], 0, 0, 0);
      }
#pragma unroll
      for (int x = 0; x < 4 * NCH; ++x)
        sc[x] = CODES ? sum_xor8(sacc[x >> 2][x & 3]) : sacc[x >> 2][x & 3];
    }
    wait_lds();  // the key slot is free
    if (more) issue_k(i + 1);
    const bool next_full = more && pages_in(i + 1) == BP;
    if (edge) {
      const int base = v0 + vpage * PAGE + slot_of(0);
      const int stop = ve - base, low = sp.low(pos) - base, sinks = sp.sinks - base;
#pragma unroll
      for (int x = 0; x < 4 * NCH; ++x) {
        const int k = (KV8 ? vt_pos(x & 12) : 8 * (x >> 2)) + (x & 3);
        sc[x] = k < stop && (k >= low || k < sinks) ? sc[x] : -__builtin_inff();
      }
    }
    float mx = -__builtin_inff();
#pragma unroll
    for (int x = 0; x < 4 * NCH; ++x) mx = fmaxf(mx, sc[x]);
    const float m_tile = max_xor32(max_xor16(mx)) * c;
    if (__builtin_amdgcn_ballot_w64(m_tile > m_run + RESCALE_LOG2)) {
      const float m_new = m_tile > m_run + RESCALE_LOG2 ? m_tile : m_run;
      const float alpha = fexp2(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int mb = 0; mb < 8; ++mb) o[mb] *= alpha;
    }
    // P^T: this lane's keys of its column, its term of each, the B operands.  Terms
    // of bf16 over 8-bit pages too: many small weights together may be the output, so
    // each keeps its own precision (e4m3 ones step by 2^-15 of the largest; the
    // widened values cost 2% of 128 decoders beside 1999 tokens, 125.4 -> 128.0 us,
    // and nothing of decoders alone, 193.6 us).
    u32x4_t pk[NCH / 2], third[NCH / 2];
#pragma unroll
    for (int w = 0; w < 2 * NCH; ++w) {
      float e0 = fexp2(__builtin_fmaf(sc[2 * w], c, -m_run));
      float e1 = fexp2(__builtin_fmaf(sc[2 * w + 1], c, -m_run));
      l_run += e0 + e1;
      if constexpr (OUT32) {
        // (Columns 8-15 have no third term: the least weight of the second.)
        const uint32_t t0 = cut(e0, e1), t1 = above_zero<KV8>(cut(e0, e1), t0);
        pk[w >> 2][w & 3] = col >= 8 ? t1 : t0;
        third[w >> 2][w & 3] = above_zero<KV8>(col >= 8 ? 0u : pack_bf16(e0, e1), t1);
      } else {
        pk[w >> 2][w & 3] = pack_term(e0, e1, col >= 8);
      }
    }
    // The values; behind them the next block's keys may be in flight.
    if (next_full)
      wait_copies<8>();
    else
      wait_copies<0>();
    if (edge) {
      // Values that the token does not see are zeroed (a probability of 0 times
      // a NaN would still be NaN).
      zero_values<KV8, BP, false>(wl + SLOT, sp, v0, pos, ve);
      wave_sync();
    }
    // O^T += V^T P^T, eight blocks of 16 dims.
    if constexpr (KV8) {
      const float vs = scale_of(etab[BP * i + vpage] >> 8);
      codes_t vc[8];
#pragma unroll
      for (int mb = 0; mb < 8; ++mb)
        vc[mb] = *reinterpret_cast<const codes_t*>(wl + vbyte + mb * 256);
#pragma unroll
      for (int mb = 0; mb < 8; ++mb) {
        bf16x8_t x[2];
        widen(vc[mb], vs, &x[0], &x[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          o[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[h], __builtin_bit_cast(bf16x8_t, pk[h]),
                                                          o[mb], 0, 0, 0);
          if constexpr (OUT32)
            o[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                x[h], __builtin_bit_cast(bf16x8_t, third[h]), o[mb], 0, 0, 0);
        }
      }
    } else {
      bf16x8_t vf[8];
#pragma unroll
      for (int mb = 0; mb < 8; ++mb)
        vf[mb] = *reinterpret_cast<const bf16x8_t*>(wl + vbyte + mb * 512);
#pragma unroll
      for (int mb = 0; mb < 8; ++mb) {
        o[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[mb], __builtin_bit_cast(bf16x8_t, pk[0]),
                                                        o[mb], 0, 0, 0);
        if constexpr (OUT32)
          o[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              vf[mb], __builtin_bit_cast(bf16x8_t, third[0]), o[mb], 0, 0, 0);
      }
    }
    wait_lds();  // the value slot is free
    if (more) issue_v(i + 1);
  }

  // Each lane group holds a quarter of its head's keys, a head's two columns a
  // term each (both the same row sum).  Then the wavefronts' results are added
  // through LDS: quad (head, 4 mb + gq) holds dims 16 mb + 4 gq .. + 3.
  const float l_tot = sum_xor32(sum_xor16(l_run));
#pragma unroll
  for (int mb = 0; mb < 8; ++mb)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[mb][i] = sum_xor8(o[mb][i]);
  wait_memory_complete();
  meet();  // every wavefront is done with its slots
  f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);
  float* stat = reinterpret_cast<float*>(smem + NW * G * 512);  // m[NW][G], l[NW][G]
  auto at = [](int w, int h, int q) { return (w * G + h) * 32 + (q ^ ((h & 7) << 2)); };
  if (col < G) {
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) red[at(wave, col, 4 * mb + gq)] = o[mb];
    if (gq == 0) {
      stat[wave * G + col] = m_run;
      stat[NW * G + wave * G + col] = l_tot;
    }
  }
  meet();
  const int slot_floats = slot_floats_for(G);
  const Slots sl = group_slots(a.ws, f[DLFP_W_WSGROUP], nsplits, slot_floats);
  const int my = f[DLFP_W_SPLIT] * slot_floats;
  // Thread: quad q4 of head h, and of heads 2 NW further with few wavefronts.
  const int q4 = tid & 31;
#pragma unroll
  for (int h0 = 0; h0 < G; h0 += 2 * NW) {
    const int h = h0 + (tid >> 5);
    if (h >= G) continue;
    float M = NEG_BIG, L = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, stat[w * G + h]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float e = fexp2(stat[w * G + h] - M);
      L += e * stat[NW * G + w * G + h];
      acc += e * red[at(w, h, q4)];
    }
    if (nsplits == 1) {
      const float inv = 1.f / L;
      store4(a, ((int64_t)tok * a.hq + kh * G + h) * D + 4 * q4, acc[0] * inv, acc[1] * inv,
             acc[2] * inv, acc[3] * inv);
    } else {
      pstore4(sl, my + h * D + 4 * q4, acc);
      if (q4 == 0) {
        pstore1(sl, my + G * D + h, M);
        pstore1(sl, my + G * D + G + h, L);
      }
    }
  }
  if (nsplits == 1) return;

  // The last arriver merges the splits in order.
  const int grp = f[DLFP_W_GROUP];
  wait_memory_complete();
  meet();  // every wave of the unit has completed its stores
  if constexpr (NW == 1) {
    int order = 0;
    if (lane == 0) order = arrive(a.ws, grp);
    if (uniform(order) != nsplits - 1) return;
  } else {
    if (tid == 0) *flag = arrive(a.ws, grp) == nsplits - 1;
    __syncthreads();
    if (!*flag) return;
  }
#pragma unroll
  for (int h0 = 0; h0 < G; h0 += 2 * NW) {
    const int h = h0 + (tid >> 5);
    if (h >= G) continue;
    // Batches of NB splits: all loads of a batch go out before any is used.
    constexpr int NB = 16;
    float M = NEG_BIG, L = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < nsplits; j += NB) {
      float mj[NB], lj[NB];
      f32x4_t x[NB];
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const int b = (j + u) * slot_floats;
        mj[u] = pload1(sl, b + G * D + h);
        lj[u] = pload1(sl, b + G * D + G + h);
        x[u] = pload4(sl, b + h * D + 4 * q4);
      }
      float mn = M;
#pragma unroll
      for (int u = 0; u < NB; ++u)
        if (j + u < nsplits) mn = fmaxf(mn, mj[u]);
      const float rs = fexp2(M - mn);
      M = mn;
      L *= rs;
      acc *= rs;
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const float e = j + u < nsplits ? fexp2(mj[u] - mn) : 0.f;
        L += e * lj[u];
        acc += e * x[u];
      }
    }
    const float inv = 1.f / L;
    store4(a, ((int64_t)tok * a.hq + kh * G + h) * D + 4 * q4, acc[0] * inv, acc[1] * inv,
           acc[2] * inv, acc[3] * inv);
  }
  if (tid == 0)
    __hip_atomic_store(group_counter(a.ws, grp), 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---------------------------------------------------------------- kernels

// The unit of workgroup b of a launch with prefill units.  The i-th prefill
// workgroup takes unit xcd_remap(i); all parts of the grid but the last begin at a
// multiple of eight, so it runs on XCD i % 8.  Workgroups go to the XCDs and to the
// four shader engines of each in turn, and wait for their own: groups of 32 give
// all of them the same order of long and short ones (in groups of eight, one
// engine got all of the prefill units, and of 512 slots 200 stood empty).
constexpr int GRID_GROUP = 32;
__device__ __forceinline__ int unit_of(const Args& a, int b) {
  const int np = a.num_prefill;
  if (b < a.lead) return xcd_remap(b, np);
  b -= a.lead;
  if (b < a.decode_lead) return np + b;
  b -= a.decode_lead;
  // (The prefill units behind decode_rest workgroups keep their XCDs together, others
  // than those of the lead where the rest is no multiple of eight.)
  if (a.decode_rest > 0)
    return b < a.decode_rest ? np + a.decode_lead + b : xcd_remap(a.lead + b - a.decode_rest, np);
  const int gp = a.prefill_groups, g = gp + a.decode_groups;
  const int group = b / GRID_GROUP, lane = b % GRID_GROUP;
  const int before = group < g ? (int)((uint64_t)group * gp / max(g, 1)) : gp;
  if (group < g) {
    const bool prefill = (int)((uint64_t)(group + 1) * gp / g) > before;
    return prefill ? xcd_remap(a.lead + GRID_GROUP * before + lane, np)
                   : np + a.decode_lead + GRID_GROUP * (group - before) + lane;
  }
  b -= GRID_GROUP * g;
  const int left = np - a.lead - GRID_GROUP * gp;
  return b < left ? xcd_remap(a.lead + GRID_GROUP * gp + b, np)
                  : np + a.decode_lead + GRID_GROUP * a.decode_groups + b - left;
}

template <int G, bool KV8, bool OUT32>
__global__ __launch_bounds__(THREADS, 2) void window_kernel(Args a) {
  __shared__ __attribute__((aligned(16))) char smem[window_lds<KV8>()];
  __shared__ int flag, special;
  const int u = unit_of(a, blockIdx.x);  // prefill unit, or num_prefill + decode workgroup
  const int32_t* rec = a.work + (int64_t)u * DLFP_WORK_INTS;
  if (u >= a.num_prefill) {
    if (a.solo) {
      const int wave = uniform(threadIdx.x >> 6), d = 4 * (u - a.num_prefill) + wave;
      if (d < a.num_units - a.num_prefill)
        decode_unit<G, KV8, OUT32, 1>(a, a.work + (int64_t)(a.num_prefill + d) * DLFP_WORK_INTS,
                                      smem + wave * decode_wave_lds<KV8, 1>(), nullptr);
    } else {
      decode_unit<G, KV8, OUT32, 4>(a, rec, smem, &flag);
    }
    return;
  }
  prompt_unit<G, KV8, OUT32>(a, load_record(rec), smem, &flag, &special);
}

template <int G, bool KV8, bool OUT32, int NW>
__global__ __launch_bounds__(NW * 64, 2) void window_decode_kernel(Args a) {
  __shared__ __attribute__((aligned(16))) char smem[NW * decode_wave_lds<KV8, NW>()];
  __shared__ int flag;
  decode_unit<G, KV8, OUT32, NW>(a, a.work + (int64_t)blockIdx.x * DLFP_WORK_INTS, smem, &flag);
}

template <int G, bool KV8, bool OUT32>
hipError_t launch_window(const Args& a, int grid, int nw, hipStream_t stream) {
  if (a.num_prefill > 0)
    window_kernel<G, KV8, OUT32><<<grid, THREADS, 0, stream>>>(a);
  else if (nw == 8)
    window_decode_kernel<G, KV8, OUT32, 8><<<a.num_units, 8 * 64, 0, stream>>>(a);
  else if (nw == 4)
    window_decode_kernel<G, KV8, OUT32, 4><<<a.num_units, 4 * 64, 0, stream>>>(a);
  else
    window_decode_kernel<G, KV8, OUT32, 1><<<a.num_units, 64, 0, stream>>>(a);
  return hipGetLastError();
}

template <int G, bool KV8>
hipError_t launch_window(const Args& a, int grid, int nw, hipStream_t stream) {
  return a.out_f32 ? launch_window<G, KV8, true>(a, grid, nw, stream)
                   : launch_window<G, KV8, false>(a, grid, nw, stream);
}

// Validation and launch shared by the two entry points.
template <bool KV8>
int attention_window(const dlfp_dims* dims, const dlfp_meta* meta, const int32_t* d_work,
                     const int32_t* d_block_table, int32_t max_blocks, int32_t num_blocks,
                     const void* q, const void* k_cache, const void* v_cache,
                     const uint8_t* k_exp, const uint8_t* v_exp, float scale, void* out,
                     int32_t out_dtype, void* workspace, size_t workspace_bytes,
                     hipStream_t stream) {
  int g = 0;
  const int st = dlfp::check_dims(dims, &g);
  if (st != DLFP_OK) return st;
  if (!meta) return DLFP_EINVAL;
  if (out_dtype != 0 && out_dtype != 1) return DLFP_EINVAL;
  if (!(scale > 0.f) || !(scale < 3.0e38f)) return DLFP_EINVAL;
  if (meta->num_units < 0 || meta->num_prefill_units < 0 ||
      meta->num_prefill_units > meta->num_units || meta->num_groups < 0 ||
      meta->num_groups > DLFP_MAX_GROUPS)
    return DLFP_EINVAL;
  if (meta->num_units == 0) return DLFP_OK;
  // The records of dlfp_build_varlen_meta have other fields.
  if (meta->decode_pages_in_flight != DLFP_WINDOW_META) return DLFP_EINVAL;
  if (meta->prefill_lead_units < 0 || meta->prefill_lead_units > meta->num_prefill_units)
    return DLFP_EINVAL;
  if (!d_work || !d_block_table || !q || !k_cache || !v_cache || !out || !workspace)
    return DLFP_EINVAL;
  if (KV8 && (!k_exp || !v_exp)) return DLFP_EINVAL;
  for (const void* p : {q, k_cache, v_cache, static_cast<const void*>(out),
                        static_cast<const void*>(workspace)})
    if (reinterpret_cast<uintptr_t>(p) % 16) return DLFP_EINVAL;
  if (max_blocks <= 0 || num_blocks <= 0) return DLFP_EINVAL;
  if ((int64_t)workspace_bytes < meta->workspace_bytes ||
      workspace_bytes < (size_t)DLFP_WORKSPACE_PARTIALS)
    return DLFP_ENOSPC;
  Args a;
  a.work = d_work;
  a.block_table = d_block_table;
  a.q = static_cast<const uint16_t*>(q);
  a.kc = static_cast<const char*>(k_cache);
  a.vc = static_cast<const char*>(v_cache);
  a.k_exp = k_exp;
  a.v_exp = v_exp;
  a.out = out;
  a.ws = static_cast<float*>(workspace);
  a.max_blocks = max_blocks;
  a.num_blocks = num_blocks;
  a.hq = dims->num_q_heads;
  a.hkv = dims->num_kv_heads;
  a.num_units = meta->num_units;
  a.num_prefill = meta->num_prefill_units;
  a.out_f32 = out_dtype;
  a.scale_log2 = scale * LOG2E;
  const int cus = dlfp::compute_units();
  const int decode_units = a.num_units - a.num_prefill;
  // Decode units of a wavefront each spend no workgroup on their start and sum, but
  // last four times as long: 29 ns a key of bf16 pages, 25 of 8-bit ones.  They are
  // - those of up to 128 KiB of cache that are more than two for each compute unit, a
  //   further round of workgroups (8-bit pages: 640 units of 64 keys 6.1 us, of four
  //   wavefronts 10.0, 2048 10.1 and 21.3, 2048 of 512 keys 44.4 and 48.3; bf16: 640
  //   of 256 keys 16.1 and 17.2, 2048 of 128 23.8 and 27.1);
  // - beside prefill units those that last up to a quarter of the launch, by its
  //   operations at 1120 TFLOP/s and its bytes at 6.4 TB/s, or 0.45 of it where the
  //   prompts are a third of it or more and hide the last of them, and every compute
  //   unit gets some (8-bit pages: 500 decoders of 64 keys beside 512 tokens 32.4 us,
  //   of four wavefronts 57.1, of 256 keys 61.4 and 77.5; 128 windowed ones of 2048
  //   keys beside 1999 tokens 128 and 140, of 1024 to 8192 keys 388 and 428; not 70 of
  //   500 keys beside 512 tokens, which last longer, 32.5 and 27.7, 32 of 2000 beside
  //   1024, 86 and 43, nor bf16, 16 of 9 to 37 thousand in 792 units beside 328, 396 and
  //   357.  The estimate leaves four wavefronts to bf16 pages of the 128 windowed ones
  //   too, 187 and 200; those of 1024 to 8192 keys are equal, 523 and 520).
  const double key_us = (KV8 ? 256 : 512) / 6.4e6, tile_key_us = 128 * 512 / 1120e6;
  const double unit_us = meta->decode_split_tokens * (KV8 ? 25e-3 : 29e-3);
  const double prefill_us = 0.85 * a.num_prefill * meta->prefill_split_tokens * tile_key_us;
  const double decode_us = 0.85 * decode_units * (double)meta->decode_split_tokens * key_us;
  const int64_t unit_bytes = (int64_t)meta->decode_split_tokens * 2 * DLFP_HEAD_DIM * (KV8 ? 1 : 2);
  const bool hidden = 2. * prefill_us >= decode_us && decode_units >= 4 * cus;
  a.solo = (decode_units > 2 * cus && unit_bytes <= 128 << 10) ||
           (a.num_prefill > 0 && unit_us <= (prefill_us + decode_us) * (hidden ? 0.45 : 0.25));
  const int decode_wgs = a.solo ? (decode_units + 3) / 4 : decode_units;
  // One prefill unit for each compute unit, then one decode unit for each, so that
  // both shares run from the start (beside each other each runs at 0.62 to 0.65 of
  // its speed alone).  A decode share that takes as long as the prefill share goes on
  // beside it: the rest of the prefill units come mixed with as many decode units
  // as take the same time, the decode units left behind them (128 windowed decoders
  // beside 1999 prompt tokens, 8-bit pages 128.6 us, without the mixture 143.5, all
  // prefill units first 159; bf16 197.5, 208 and 243).  A shorter one would leave
  // the last prefill units alone: they come first then (whole contexts, 8-bit
  // pages: 403 us, mixed 475).  The last of up to `cus` decode workgroups, less than a
  // group, go in front of them too, so that a few are not left to the end (2 decoders
  // beside 1408 tokens of 64 heads, bf16: 48 us, behind them 58).
  a.lead = a.num_prefill;
  a.decode_lead = a.decode_rest = a.prefill_groups = a.decode_groups = 0;
  if (meta->prefill_lead_units < a.num_prefill && decode_wgs > 0) {
    a.lead = meta->prefill_lead_units / GRID_GROUP * GRID_GROUP;
    a.decode_lead = std::min(decode_wgs, cus) / GRID_GROUP * GRID_GROUP;
    if (decode_wgs <= cus) a.decode_rest = decode_wgs % GRID_GROUP;
    a.prefill_groups = (a.num_prefill - a.lead) / GRID_GROUP;
    // Keys of the decode units for one of the prefill units, times what a key takes
    // of the decode share alone (its bytes at 6.4 TB/s) over the prefill share alone
    // (128 rows at 1.12 PFLOP/s).
    const double key = key_us / tile_key_us;
    const double shares = meta->num_waiting_units / 1024. * key;
    const double groups = shares >= 0.9 ? 0.85 * key * a.prefill_groups * meta->prefill_split_tokens /
                                              std::max(meta->decode_split_tokens, 64) /
                                              (a.solo ? 4 : 1)
                                        : 0.;
    a.decode_groups = (int)std::min<double>((decode_wgs - a.decode_lead) / GRID_GROUP, groups);
  }
  // Wavefronts of a decode unit in a launch of decode units alone.  Eight, with long
  // units on a quarter of the compute units: one lasts as long as its chain of steps
  // (8 units of 2048 keys, 8 bits: 14.7 us, with four 16.6; bf16 13.2 and 18.3).  Else
  // four, two workgroups on a compute unit, one's start and sum behind the other (512
  // units of 1024 keys, 8 bits: 24.8 us, with eight 27.6, with one 29.4).
  const int nw = a.solo ? 1 : a.num_units <= cus / 4 && meta->decode_split_tokens > 256 ? 8 : 4;
  const int grid = a.num_prefill + decode_wgs;
  (void)hipGetLastError();
  hipError_t e;
  switch (g) {
    case 1: e = launch_window<1, KV8>(a, grid, nw, stream); break;
    case 2: e = launch_window<2, KV8>(a, grid, nw, stream); break;
    case 4: e = launch_window<4, KV8>(a, grid, nw, stream); break;
    default: e = launch_window<8, KV8>(a, grid, nw, stream); break;
  }
  return e == hipSuccess ? DLFP_OK : DLFP_EHIP;
}

}  // namespace

#endif  // DLFP_ATTENTION_WINDOW_H
