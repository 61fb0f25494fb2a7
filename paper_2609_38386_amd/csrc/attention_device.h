// Device functions that the attention kernels share: wavefront exchanges, LDS
// copies, the exchange of split-K partial results and their merges.  The merges
// and stores take any argument struct A with the fields out, out_f32, ws and hq.
#ifndef DLFP_ATTENTION_DEVICE_H
#define DLFP_ATTENTION_DEVICE_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dlfp.h"
#include "dlfp_internal.h"

namespace {

constexpr int D = DLFP_HEAD_DIM;
constexpr int PAGE = DLFP_PAGE_SIZE;
constexpr int PAGE_ELEMS = PAGE * D;          // elements of a (block, head) page

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

constexpr float NEG_BIG = -1.0e30f;
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a),
                                         __builtin_bit_cast(bf16x2_t, b), c, false);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2_t v;
  v[0] = (__bf16)lo;
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}

// A probability in two bf16 terms, for products whose columns come in pairs: the
// upper half, cut off, or (`low`) the rest, which is then positive; at least the
// least normal number, so that the product with an infinite value is that
// infinity in both.
__device__ __forceinline__ uint32_t pack_term(float p0, float p1, bool low) {
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
  const uint32_t b0 = __builtin_bit_cast(uint32_t, p0), b1 = __builtin_bit_cast(uint32_t, p1);
  const uint32_t upper = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
  const uint32_t rest = pack_bf16(p0 - __builtin_bit_cast(float, b0 & 0xFFFF0000u),
                                  p1 - __builtin_bit_cast(float, b1 & 0xFFFF0000u));
  const u16x2_t least = {0x0080, 0x0080};
  const u16x2_t kept = __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, rest), least);
  return low ? __builtin_bit_cast(uint32_t, kept) : upper;
}
// x plus the x of lane ^ 8 (rows of 16 lanes rotated by 8).  The sum is made
// here and not where its lanes are used, which keeps it one instruction.
__device__ __forceinline__ float sum_xor8(float x) {
  float y = x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x128,
                                                                   0xF, 0xF, true));
  asm volatile("" : "+v"(y));
  return y;
}

__device__ __forceinline__ float fexp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float shfl_xor(float x, int m) { return __shfl_xor(x, m); }

// Combine a value with the one of lane ^ 16 (or lane ^ 32) by the gfx950
// permlane swaps (VALU, no LDS round trip): swapping two copies of a value
// leaves the lane's own value in one register and its partner's in the
// other.  Written as assembly because the compiler reads both results of
// the swap builtin from one register, losing the partner's value.
__device__ __forceinline__ void swap16(float& a, float& b) {
  asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
}
__device__ __forceinline__ void swap32(float& a, float& b) {
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
}
__device__ __forceinline__ float max_xor16(float x) {
  float a = x, b = x;
  swap16(a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float max_xor32(float x) {
  float a = x, b = x;
  swap32(a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float sum_xor16(float x) {
  float a = x, b = x;
  swap16(a, b);
  return a + b;
}
__device__ __forceinline__ float sum_xor32(float x) {
  float a = x, b = x;
  swap32(a, b);
  return a + b;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Work records are read-only for the launch: read through the constant
// address space, so that a wave-uniform record comes in with scalar loads
// (one round trip for all its fields).
typedef const __attribute__((address_space(4))) int32_t* record_ptr;
__device__ __forceinline__ record_ptr as_record(const int32_t* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (record_ptr)(((uint64_t)hi << 32) | lo);
}
// A whole record in one scalar load.
typedef int32_t record_t __attribute__((ext_vector_type(16), aligned(4)));
__device__ __forceinline__ record_t load_record(const int32_t* p) {
  return *(const __attribute__((address_space(4))) record_t*)as_record(p);
}

// Lanes of one wavefront hand data to each other through LDS.  The hardware
// runs a wave's LDS operations in order; this keeps the compiler from moving a
// lane's LDS accesses across the hand-off (it reasons per lane, so a store to
// an address the lane itself never reads would otherwise be free to move).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ int* group_counter_ptr(float* ws, int grp) {
  return reinterpret_cast<int*>(reinterpret_cast<char*>(ws) + DLFP_WORKSPACE_HEADER) + grp;
}

// Error word values: 1 = a block id outside the pool, 2 = a wait for the
// append records ran out.
__device__ __forceinline__ void raise_error(float* ws, int code = 1) {
  __hip_atomic_store(reinterpret_cast<int*>(ws), code, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Split-K partial results cross workgroups (and XCDs, whose L2s are not
// coherent with each other).  They are written with device-coherent stores
// (the sc1 policy: written through to the device coherence point) and read
// back with device-coherent loads (which do not return stale L2 lines), both
// through a buffer resource bounded to the group's slots.  Before a unit
// bumps its group counter it waits until all its vector-memory operations,
// stores included, have completed; the last arriver issues its loads only
// after the counter read has returned.  This orders the exchange without
// writing back or invalidating whole L2 caches per unit.
constexpr int CPOL_SC1 = 16;  // cache-policy bit: coherent at device scope

// Loads past the group's slots return zero: a batch of a decode merge may reach
// past the last split (a repeated split with a weight of zero would make an
// infinite partial value a NaN, as the masked keys of a prefill tile make one).
struct Slots {
  __amdgpu_buffer_rsrc_t r;
};

__device__ __forceinline__ Slots group_slots(float* ws, int group_off, int nsplits,
                                             int slot_floats) {
  return Slots{__builtin_amdgcn_make_buffer_rsrc(ws + group_off, 0, nsplits * slot_floats * 4,
                                                 0x00020000)};
}
__device__ __forceinline__ void pstore4(Slots s, int float_off, f32x4_t v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), s.r, float_off * 4, 0,
                                         CPOL_SC1);
}
__device__ __forceinline__ void pstore2(Slots s, int float_off, f32x2_t v) {
  __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2_t, v), s.r, float_off * 4, 0,
                                        CPOL_SC1);
}
__device__ __forceinline__ void pstore1(Slots s, int float_off, float v) {
  __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), s.r, float_off * 4, 0,
                                        CPOL_SC1);
}
__device__ __forceinline__ f32x4_t pload4(Slots s, int float_off) {
  return __builtin_bit_cast(f32x4_t,
                            __builtin_amdgcn_raw_buffer_load_b128(s.r, float_off * 4, 0, CPOL_SC1));
}
__device__ __forceinline__ f32x2_t pload2(Slots s, int float_off) {
  return __builtin_bit_cast(f32x2_t,
                            __builtin_amdgcn_raw_buffer_load_b64(s.r, float_off * 4, 0, CPOL_SC1));
}
__device__ __forceinline__ float pload1(Slots s, int float_off) {
  return __builtin_bit_cast(float,
                            __builtin_amdgcn_raw_buffer_load_b32(s.r, float_off * 4, 0, CPOL_SC1));
}
// Floats per partial slot: O (rows x 128), m[rows], l[rows], padded to 256 bytes.
__device__ __forceinline__ int slot_floats_for(int rows) {
  return (rows * (D + 2) + 63) / 64 * 64;
}
// Wait for every outstanding vector-memory operation of this wave (on gfx9 the
// vector-memory counter covers stores) and keep the compiler from moving
// memory operations across the wait.
__device__ __forceinline__ void wait_memory_complete() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0), expcnt and lgkmcnt unconstrained
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}
// Wait until at most N of this wave's copies are in flight; until its LDS
// reads have returned.
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ int arrive(float* ws, int grp) {
  return __hip_atomic_fetch_add(group_counter_ptr(ws, grp), 1, __ATOMIC_RELAXED,
                                __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ int* group_counter(float* ws, int grp) {
  return group_counter_ptr(ws, grp);
}

// Workgroups are dealt round-robin over the 8 XCDs; map them so that each XCD
// gets a contiguous range of prefill units (same KV head -> same L2).
__device__ __forceinline__ int xcd_remap(int b, int n) {
  const int x = b & 7, i = b >> 3;
  const int per = n >> 3, rem = n & 7;
  return x * per + min(x, rem) + i;
}

// Store 4 consecutive output values of one row.
template <class A>
__device__ __forceinline__ void store4(const A& a, int64_t elem, float v0, float v1, float v2,
                                       float v3) {
  if (a.out_f32) {
    f32x4_t v = {v0, v1, v2, v3};
    *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + elem) = v;
  } else {
    u32x2_t v = {pack_bf16(v0, v1), pack_bf16(v2, v3)};
    *reinterpret_cast<u32x2_t*>(static_cast<uint16_t*>(a.out) + elem) = v;
  }
}

template <class A>
__device__ __forceinline__ void store2(const A& a, int64_t elem, float v0, float v1) {
  if (a.out_f32) {
    f32x2_t v = {v0, v1};
    *reinterpret_cast<f32x2_t*>(static_cast<float*>(a.out) + elem) = v;
  } else {
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + elem) = pack_bf16(v0, v1);
  }
}

// A running row maximum is only raised once a tile's maximum exceeds it by
// more than this many powers of two, so probabilities stay below 2^8 and the
// accumulators are rescaled rarely (the final division by the row sum makes
// the result independent of the reference maximum).
constexpr float RESCALE_LOG2 = 8.f;

// V^T rows (dims) store their two 16-byte halves swapped when bits 2 and 3
// of the dim differ; 8 (or 16) consecutive dims then cover every LDS bank
// once for each half.
__device__ __forceinline__ int vt_swz(int d) { return ((d >> 2) ^ (d >> 3)) & 1; }

// Position of token slot t inside a V^T row of the cache: slots 4-7 and 8-11
// trade places (bits 2 and 3 swap), matching the key order of the
// S^T accumulator rows that become the PV operand.
__device__ __forceinline__ int vt_pos(int t) { return (t & 3) | ((t & 4) << 1) | ((t & 8) >> 1); }

typedef __attribute__((address_space(3))) char* lds_ptr_t;
// One 16-byte piece per lane, global to LDS without registers: lane l's piece
// lands at LDS byte address lds + 16 l (lds is wave-uniform).  Completion is
// counted by the vector-memory counter; the caller waits for it explicitly
// (wait_memory_complete) before the barrier that publishes the tile.  The
// copy is written as assembly so that the compiler, which cannot tell the
// ring slots apart, does not wait for it before every LDS read.
__device__ __forceinline__ void lds_copy16(const char* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(src), "s"(lds)
               : "memory", "m0");
}
// The same copy from a wave-uniform base and a lane's byte offset (the address
// costs no vector instruction).
__device__ __forceinline__ const char* uniform_ptr(const void* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const char*>(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ void lds_copy16(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(lds)
               : "memory", "m0");
}
// The same copy marked non-temporal, for the decode share's pages: each is
// read once per launch, so streaming them past the caches keeps the prefill
// share's K/V tiles (read by many query tiles) resident in L2 and raises the
// decode share's own HBM rate (Qwen3-32B decode-only 5.91 -> 6.49 TB/s).
__device__ __forceinline__ void lds_copy16_nt(const char* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt"
               :
               : "v"(src), "s"(lds)
               : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_addr(char* p) {
  return (uint32_t)(uintptr_t)(lds_ptr_t)p;
}

// Keep the elements of a 16-bit-element vector whose key index is below
// limit; key_of(e) gives element e's key.
template <typename F>
__device__ __forceinline__ u32x4_t mask_elems(u32x4_t v, int limit, F key_of) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t lo = key_of(2 * w) < limit ? 0x0000FFFFu : 0u;
    const uint32_t hi = key_of(2 * w + 1) < limit ? 0xFFFF0000u : 0u;
    v[w] &= (lo | hi);
  }
  return v;
}

// Last arriver's merge of a prefill group: every split's (O, m, l) in split
// order with an online rescale.  TPR threads per row; a row's 128 values are
// 32 four-float pieces (chunk c = piece / 2, half = piece % 2 of the partial
// layout), and the thread with index sub in its row takes pieces
// sub + TPR i.  The loads of NB splits (pieces, maxima and sums) are issued
// before any is consumed, so a batch costs about one memory round trip; NB is
// chosen so that a batch holds about 136 registers.  Every load instruction
// of a wavefront reads whole contiguous runs of the partial layout.
// A batch that reaches past the last split takes that one again with a weight of
// zero, which makes a NaN of an infinite partial value; with EXACT it leaves it out.
template <int G, int TPR, class A, bool EXACT = false>
__device__ __forceinline__ void prefill_merge(const A& a, const Slots sl, int slot_floats,
                                              int nsplits, int rows, int row0, int kh) {
  constexpr int NP = 32 / TPR;             // pieces per thread
  constexpr int PP = NP < 8 ? NP : 8;      // pieces per pass
  constexpr int PASSES = NP / PP;
  constexpr int NB = 32 / PP;              // splits per batch
  const int tid = threadIdx.x;
  if (tid >= TPR * rows) return;
  const int row = tid / TPR, sub = tid % TPR;
  const int64_t orow = ((int64_t)(row0 + row / G) * a.hq + kh * G + row % G) * D;
  for (int pass = 0; pass < PASSES; ++pass) {
    float M = NEG_BIG, lsum = 0.f;
    f32x4_t acc[PP];
#pragma unroll
    for (int i = 0; i < PP; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < nsplits; j += NB) {
      float mj[NB], lj[NB];
      f32x4_t x[NB][PP];
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const int b = min(j + u, nsplits - 1) * slot_floats;
        mj[u] = pload1(sl, b + rows * D + row);
        lj[u] = pload1(sl, b + rows * D + rows + row);
#pragma unroll
        for (int i = 0; i < PP; ++i) {
          const int piece = sub + TPR * (pass * PP + i);
          x[u][i] = pload4(sl, b + (((piece >> 1) * rows + row) * 8 + 4 * (piece & 1)));
        }
      }
      float mn = M;
#pragma unroll
      for (int u = 0; u < NB; ++u)
        if (j + u < nsplits) mn = fmaxf(mn, mj[u]);
      const float rs = fexp2(M - mn);
      M = mn;
      lsum *= rs;
#pragma unroll
      for (int i = 0; i < PP; ++i) acc[i] *= rs;
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        if (EXACT && j + u >= nsplits) break;
        const float w = j + u < nsplits ? fexp2(mj[u] - mn) : 0.f;
        lsum += w * lj[u];
#pragma unroll
        for (int i = 0; i < PP; ++i) acc[i] += w * x[u][i];
      }
    }
    const float inv = 1.f / lsum;
#pragma unroll
    for (int i = 0; i < PP; ++i) {
      // piece -> chunk c = 4 mb + g4 and half h -> dims 32 mb + 8 g4 + 4 h
      const int piece = sub + TPR * (pass * PP + i);
      const int c = piece >> 1;
      const int dim = 32 * (c >> 2) + 8 * (c & 3) + 4 * (piece & 1);
      store4(a, orow + dim, acc[i][0] * inv, acc[i][1] * inv, acc[i][2] * inv, acc[i][3] * inv);
    }
  }
}

// Last arriver of a decode split group: merges the group's partial results
// (O[G][128], m[G], l[G] per split, in split order) into the output.  Lane
// `lane` writes dims 2 lane and 2 lane + 1 of every head; obase is the
// element offset of those dims of the group's first head.
template <int G, class A>
__device__ __forceinline__ void decode_merge(const A& a, const Slots sl, int slot_floats,
                                             int nsplits, int64_t obase, int grp) {
  const int lane = threadIdx.x & 63;
  // Entry f = j G + h stands for head h of split j.  Per batch
  // of up to 64 entries, lane e loads entry e's maximum and row sum while
  // every lane loads its two dims of the batch's entries (in groups of 16,
  // only as many groups as the batch has entries), so a batch costs one
  // memory round trip; the running per-head maximum rescales what earlier
  // batches summed, and entries are accumulated in split order.
  const int nf = nsplits * G;
  float M[G], lsum[G], acc0[G], acc1[G];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    M[h] = NEG_BIG;
    lsum[h] = acc0[h] = acc1[h] = 0.f;
  }
  for (int f0 = 0; f0 < nf; f0 += 64) {
    const int n = min(64, nf - f0);
    const int fl = f0 + lane;
    const int lbase = (fl / G) * slot_floats + G * D + fl % G;
    const float mf = lane < n ? pload1(sl, lbase) : NEG_BIG;
    const float lf = pload1(sl, lbase + G);
    f32x2_t v[4][16];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (16 * q < n) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int fe = f0 + 16 * q + e;
          v[q][e] = pload2(sl, (fe / G) * slot_floats + (fe % G) * D + 2 * lane);
        }
      }
    }
    // Batch maximum of head lane % G (f0 is a multiple of 64, so entry
    // f0 + e belongs to head e % G).
    float bm = mf;
#pragma unroll
    for (int sh = G; sh < 64; sh <<= 1) bm = fmaxf(bm, shfl_xor(bm, sh));
    float mh = NEG_BIG;
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const float mnew = fmaxf(M[h], __builtin_bit_cast(float, __builtin_amdgcn_readlane(
                                                                  __builtin_bit_cast(int, bm), h)));
      const float rs = fexp2(M[h] - mnew);
      M[h] = mnew;
      lsum[h] *= rs;
      acc0[h] *= rs;
      acc1[h] *= rs;
      if (lane % G == h) mh = mnew;
    }
    const float wf = lane < n ? fexp2(mf - mh) : 0.f;
    const float wl = wf * lf;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (16 * q < n) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int src = 16 * q + e;  // weights of entries past the batch are zero
          const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(
                                                        __builtin_bit_cast(int, wf), src));
          const float lw = __builtin_bit_cast(float, __builtin_amdgcn_readlane(
                                                         __builtin_bit_cast(int, wl), src));
          lsum[e % G] += lw;
          acc0[e % G] += w * v[q][e][0];
          acc1[e % G] += w * v[q][e][1];
        }
      }
    }
  }
#pragma unroll
  for (int h = 0; h < G; ++h) {
    const float inv = 1.f / lsum[h];
    store2(a, obase + h * D, acc0[h] * inv, acc1[h] * inv);
  }
  if (lane == 0)
    __hip_atomic_store(group_counter(a.ws, grp), 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace

#endif  // DLFP_ATTENTION_DEVICE_H
