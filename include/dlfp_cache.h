/*
 * dlfp_cache.h -- C ABI of libdlfp beside dlfp.h: the cache append with the
 * position rotation applied on the way, pages held in 8 bits, and attention
 * with a sliding window and sinks.
 *
 * One layer of a mixed iteration (Sec. 2.1) is then
 *
 *   dlfp_build_window_meta   host: packed-batch metadata and the work list
 *   dlfp_rope_append         device: rotate queries and keys, write the pages
 *   dlfp_attention_window    device: one launch of attention for all rows
 *
 * with bf16 pages, or dlfp_rope_append_kv8 and dlfp_attention_kv8 with 8-bit
 * pages.  The conventions of dlfp.h hold for every call: status codes, no
 * exceptions, nothing allocated, stream-ordered launches, arguments checked
 * before anything is launched, no work launches nothing and may pass null
 * device pointers.  The current device is the one that the stream and every
 * buffer belong to.
 *
 * bf16 pages are those of dlfp.h.  8-bit pages (half the bytes):
 *  - k_cache     [num_blocks][Hkv][16][128]   e4m3 codes, 16 token rows
 *  - v_cache     [num_blocks][Hkv][128][16]   e4m3 codes, one 16-byte row per
 *                                             dimension, slot t at position
 *                                             pi(t) as in dlfp.h
 *  - k_exp,v_exp [num_blocks][Hkv] uint8      exponent byte of a page: a code c
 *                                             stands for c * 2^(byte - 127)
 *  e4m3 is the OCP format (4 exponent bits of bias 7, 3 mantissa bits, largest
 *  value 448, no infinity, 0x7F and 0xFF NaN).  With power-of-two scales every
 *  value of a page is a bf16 number, so that attention over 8-bit pages is
 *  attention over bf16 pages of those values.  Bytes 27 (2^-100) to 240 are
 *  what the append writes for bf16 inputs below 2^120; attention takes any byte
 *  from 10 to 238 exactly (a value outside bf16's normal range is not kept).
 */
#ifndef DLFP_CACHE_H
#define DLFP_CACHE_H

#include "dlfp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ append */

/* Rotary position embedding: of a head's first rotary_dim = r dimensions, pair
 * i < r / 2 turns by the angle of the token's position: dims (i, i + r / 2), or
 * (2 i, 2 i + 1) when interleaved.  (a, b) becomes (a c - b s, b c + a s) with
 * c = table[pos][i], s = table[pos][r / 2 + i]; dims from r on stay. */
typedef struct {
  const float* table;   /* device [positions][rotary_dim]: cosines, then sines; 16-byte aligned */
  int32_t positions;    /* rows of the table */
  int32_t rotary_dim;   /* 32, 64 or 128 */
  int32_t interleaved;  /* 0 or 1 */
} dlfp_rope;

/* Rotate the queries and keys of num_tokens new tokens to their positions and
 * write keys and values into bf16 pages, in one launch.
 *
 * positions, slot_mapping: device int32 [num_tokens]; q, k_new, v_new: device
 * bf16, token t's heads at q + t * ldq ([Hq][128]), k_new + t * ldk and
 * v_new + t * ldv ([Hkv][128]), so that the three may be parts of one
 * projection's rows; q_out: device bf16, token t's rotated heads at
 * q_out + t * ldo.  q_out may be q itself with ldo = ldq; otherwise no output
 * overlaps an input.  Strides are in elements, multiples of 8 and at least the
 * heads' 128 each; buffers are 16-byte aligned.
 *
 * The rotation is computed in fp32 (two products and a sum, each rounded) and
 * rounded once to bf16; values are copied.  A slot outside
 * [0, num_blocks * 16) leaves the pages as they are (the query is still
 * rotated); a token whose position is outside [0, positions) is left out
 * altogether.  Of two tokens with one slot, the key of either and the value of either
 * may be kept.
 * Errors: DLFP_EINVAL, DLFP_EUNSUPPORTED (dims, rotary_dim), DLFP_ERANGE (2^32
 * threads or more, of which a token has 16 for each KV head and 64 for each group of
 * 16 query heads), DLFP_EHIP. */
int dlfp_rope_append(const dlfp_dims* dims, const dlfp_rope* rope, int32_t num_tokens,
                     const int32_t* positions, const int32_t* slot_mapping, const void* q,
                     int64_t ldq, const void* k_new, int64_t ldk, const void* v_new, int64_t ldv,
                     void* q_out, int64_t ldo, void* k_cache, void* v_cache, int32_t num_blocks,
                     hipStream_t stream);

/* The same into 8-bit pages.  The tokens that a call writes to one page lie
 * within 16 rows, in ascending order of their slots, as a sequence's new tokens
 * do (another order gives undefined values in that page).  Consecutive slots of a
 * page in consecutive rows are a run; for each run (one after the other where a
 * token left out makes two of a page), KV head, and keys and values apart:
 *   amax = the largest finite magnitude among the run's tokens (keys: after the
 *          rotation, in fp32)
 *   E    = the least integer >= -100 with amax <= 448 * 2^E; when the run's
 *          first slot is not slot 0, at least the page's exponent
 * New tokens get the codes nearest to x * 2^-E (ties to even; NaN and
 * infinities become NaN); if E is larger than the page's exponent F and the
 * first slot is not 0, the slots before the first are rewritten with the codes
 * nearest to code * 2^(F - E).  Slots after the last keep their codes.  So a
 * token at slot 0 begins its page anew, whatever the page held.
 * Errors: as dlfp_rope_append. */
int dlfp_rope_append_kv8(const dlfp_dims* dims, const dlfp_rope* rope, int32_t num_tokens,
                         const int32_t* positions, const int32_t* slot_mapping, const void* q,
                         int64_t ldq, const void* k_new, int64_t ldk, const void* v_new,
                         int64_t ldv, void* q_out, int64_t ldo, void* k_cache, void* v_cache,
                         uint8_t* k_exp, uint8_t* v_exp, int32_t num_blocks, hipStream_t stream);

/* --------------------------------------------------------------- attention */

/* Which keys a row sees: at position p, key j <= p with p - j < window, or
 * j < sinks (the sequence's first tokens).  Every row sees its own key. */
typedef struct {
  int32_t window;  /* >= 1 */
  int32_t sinks;   /* >= 0 */
} dlfp_window;

/* Fields of a work record of dlfp_build_window_meta that differ from those of
 * dlfp_build_varlen_meta (dlfp.h).  A unit reads the pages that hold a key some
 * row of it sees: the first ceil(SINKS / 16) pages of the sequence, then, GAP
 * pages further, those from its first row's window on (GAP 0: every page from
 * the first).  KVBEGIN and KVEND count keys with the gap left out. */
enum {
  DLFP_W_WINDOW = 9, /* window, INT32_MAX without one (WSOFF there) */
  DLFP_W_SINKS = 14, /* sinks (PAGE0 there) */
  DLFP_W_GAP = 15    /* pages left out after the sink pages (PAGE1 there) */
};
/* decode_pages_in_flight of such a metadata, by which the attention calls know
 * it: each kind of metadata is refused where the other belongs. */
#define DLFP_WINDOW_META 3

/* dlfp_build_varlen_meta for dlfp_attention_window and dlfp_attention_kv8: the
 * same arrays and counts (num_append is 0, the two split counts are the
 * keys of the longest unit of each kind, num_waiting_units is the decode share's
 * keys over the prefill share's times 1024).  window may
 * be null: every key up to a row's own.  Only the pages that a row sees, and
 * those of the new tokens, need a block id in [0, num_blocks); other entries of
 * the block table are not read (a window's dropped pages may be -1).
 * prefill_tile_tokens, the two splits, target_units and prefill_lead_units of
 * the tuning act as in dlfp.h; splits are cut from the keys that are read.
 * Zero fields of the tuning choose by estimates of the launch time: prompts in
 * tiles of 128 rows or of 32 and in equal parts of at least 256 keys, decoders in
 * equal parts of at least 128.
 * Errors: as dlfp_build_varlen_meta; DLFP_EINVAL for a window below 1 or sinks
 * below 0; DLFP_ERANGE also for a sequence that reads more than 2^31 - 65 keys, or
 * whose splits leave a group 2 GiB of partial results or more (a tuning of short
 * splits over millions of keys); DLFP_ENOSPC also when host memory runs out. */
int dlfp_build_window_meta(const dlfp_dims* dims, const dlfp_tuning* tuning,
                           const dlfp_window* window, int32_t num_seqs, const int32_t* q_len,
                           const int32_t* kv_len, const int32_t* block_table, int32_t max_blocks,
                           int32_t num_blocks, dlfp_meta* meta);

/* One launch of masked softmax attention over bf16 pages for every new token of
 * the batch, whose keys and values are in the pages already: for query row i of
 * sequence s at position p = q_pos0[s] + i and query head h with KV head h / g,
 * out = softmax_j(scale * q.k_j) v_j over the keys j that the row sees.
 * Arguments as for dlfp_attention_mixed, with a metadata of
 * dlfp_build_window_meta; q, caches, out and workspace are 16-byte aligned.
 * Scores, statistics and sums are fp32.  With bf16 output the probabilities of a
 * prompt's rows are rounded to bf16 for the product with the values (1.1e-3 to
 * 1.6e-3 of a row in the 2-norm, below the output's own rounding) and a decoder's
 * taken in two bf16 terms; with fp32 output they are three terms, 24 bits.
 * What a row does not see changes none of its outputs, whatever it holds.  An
 * infinite value that a row sees makes that dim of its heads that infinity (or NaN,
 * if its weight is below 2^-126 of the largest), a NaN a NaN.  The units of a prompt
 * that meet one do their work twice.
 * Errors: as dlfp_attention_mixed; DLFP_EINVAL for the other kind of metadata. */
int dlfp_attention_window(const dlfp_dims* dims, const dlfp_meta* meta, const int32_t* d_work,
                          const int32_t* d_block_table, int32_t max_blocks, int32_t num_blocks,
                          const void* q, const void* k_cache, const void* v_cache, float scale,
                          void* out, int32_t out_dtype, void* workspace, size_t workspace_bytes,
                          hipStream_t stream);

/* The same over 8-bit pages and their exponents, with or without a window.  With
 * bf16 output the scores come from products of 8-bit numbers: a query is the sum
 * of two e4m3 codes in scales 2^4 apart (what lies below 2^-22 of its row's
 * largest is lost) and the matrix cores add a product's terms to within 2^-15 of
 * the sum of their magnitudes (2e-6 on average).  Probabilities are those of
 * dlfp_attention_window. */
int dlfp_attention_kv8(const dlfp_dims* dims, const dlfp_meta* meta, const int32_t* d_work,
                       const int32_t* d_block_table, int32_t max_blocks, int32_t num_blocks,
                       const void* q, const void* k_cache, const void* v_cache,
                       const uint8_t* k_exp, const uint8_t* v_exp, float scale, void* out,
                       int32_t out_dtype, void* workspace, size_t workspace_bytes,
                       hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DLFP_CACHE_H */
