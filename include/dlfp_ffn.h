/*
 * dlfp_ffn.h -- C ABI of libdlfp beside dlfp.h: projections with 4-bit weights
 * and the gated feed-forward projection.
 *
 * The cost of an iteration's linear layers (Eq. 1, Sec. 2.1) with few tokens is
 * the bytes of their weights.  A layer's weights may be kept in 4 bits, and its
 * feed-forward block is two calls:
 *
 *   dlfp_gated_linear_bf16 or dlfp_gated_linear_w4   gate, up, activation, product
 *   dlfp_linear_bf16 or dlfp_linear_w4               down
 *
 * The conventions of dlfp.h hold for every call: status codes, no exceptions,
 * nothing allocated, stream-ordered launches, arguments checked before anything
 * is launched, no tokens launch nothing and may pass null device pointers.  The
 * current device is the one that the stream and every buffer belong to.  No
 * output overlaps an input.
 *
 * 4-bit weights (17/32 byte a weight) of a layer [n][k], a row for each output
 * feature:
 *  - codes  [n][k / 2]   e2m1, two to a byte, the even column in the low half:
 *                        bit 3 the sign, bits 0-2 the magnitudes 0, 0.5, 1, 1.5,
 *                        2, 3, 4, 6
 *  - exps   [n][k / 32]  uint8, exponent byte of 32 columns of a row: a code c
 *                        stands for c * 2^(byte - 127)
 *  These are the OCP microscaling FP4 format's elements and scales.  With
 *  power-of-two scales every weight is a bf16 number for bytes 0 to 252, so that
 *  a projection with 4-bit weights is one with the bf16 weights of those values.
 *  Byte 255 makes the group's 32 weights NaN; with 253 and 254 the values from
 *  2^128 on are infinite.
 */
#ifndef DLFP_FFN_H
#define DLFP_FFN_H

#include "dlfp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Columns of a row that share an exponent byte. */
#define DLFP_W4_GROUP 32

/* Weights to 4 bits.  w: device bf16, row i at w + i * ldw (ldw >= k, a multiple
 * of 8, w 16-byte aligned); codes (16-byte aligned), exps: device, as above.
 * A group's exponent is the least, from -125 to 125, that leaves its largest
 * magnitude at 6 or below (byte 2 to 252); codes are the nearest ones, ties to
 * even, past 6 (only at exponent 125) they stay 6, and keep the sign of w, of
 * zeros too.  A group with an infinite or NaN value gets byte 255 and codes 0.
 * k is a multiple of 32 (DLFP_EUNSUPPORTED); n = 0 launches nothing.
 * Errors: DLFP_EINVAL, DLFP_EUNSUPPORTED, DLFP_ERANGE (2^34 weights or more),
 * DLFP_EHIP. */
int dlfp_quantize_w4(int32_t n, int32_t k, const void* w, int64_t ldw, void* codes, void* exps,
                     hipStream_t stream);

/* The values of 4-bit weights, in bf16: row i at w + i * ldw (ldw >= k, a multiple
 * of 8, w 16-byte aligned).  Errors as dlfp_quantize_w4. */
int dlfp_dequantize_w4(int32_t n, int32_t k, const void* codes, const void* exps, void* w,
                       int64_t ldw, hipStream_t stream);

/* Projection with 4-bit weights W:
 *   out[i][j] = sum_l x[i][l] * W[j][l],  i < m, j < n, l < k
 * x: device bf16, row i at x + i * ldx (ldx >= k, a multiple of 8, x 16-byte
 * aligned); codes, exps (16-byte aligned): device, as above; out: device, row i
 * at out + i * ldo (ldo >= n, a multiple of 4), out_dtype 0 = bf16 (8-byte
 * aligned), 1 = fp32 (16-byte aligned).  Products are exact, sums are fp32 in an
 * order that depends on m, n, k and the workspace, and are rounded once.  n must be a
 * multiple of 16 and k of 64 (DLFP_EUNSUPPORTED otherwise); m = 0 launches nothing.
 *
 * workspace: device, 16-byte aligned, or null: where there are few tiles, K is split over
 * workgroups, whose partial sums pass through it into a second launch.  How many bytes the
 * fastest form takes dlfp_projection_workspace says; with fewer (0 with null) a form that
 * fits is taken.  It overlaps no other buffer, and its contents matter neither before
 * nor after; calls that may overlap (on two streams, or as parts of graphs that may) need
 * workspaces of their own.
 * Errors: DLFP_EINVAL, DLFP_EUNSUPPORTED, DLFP_ERANGE (more than 2^31 - 1025 tokens or
 * features, 2^39 outputs or more, or 2^32 threads or more in every form of the call: there is
 * one of 512 threads for each 256 tokens and 256 features (gated: 128); with rows 2^22 elements
 * or more apart there is only one of 512 for each 16 and 16, gated with bf16 weights of 256 for
 * each 64 and 32), DLFP_EHIP (of the second launch: the first stays enqueued). */
int dlfp_linear_w4(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx, const void* codes,
                   const void* exps, void* out, int64_t ldo, int32_t out_dtype, void* workspace,
                   size_t workspace_bytes, hipStream_t stream);

/* Activations of the gated projection. */
#define DLFP_SILU 0 /* g / (1 + e^-g) */
#define DLFP_GELU 1 /* g / (1 + e^(-2 t)), t = sqrt(2 / pi) (g + 0.044715 g^3): the tanh form */

/* Gate, up, activation and product of a feed-forward block:
 *   out[i][j] = act(sum_l x[i][l] * G[j][l]) * sum_l x[i][l] * U[j][l]
 * with bf16 weights w_gate, w_up: device [n][k], 16-byte aligned (halves of one
 * [2 n][k] buffer, in either order, or two buffers).  Sums, activation and product
 * are fp32 and are rounded once.  The rest as dlfp_linear_w4. */
int dlfp_gated_linear_bf16(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                           const void* w_gate, const void* w_up, int32_t activation, void* out,
                           int64_t ldo, int32_t out_dtype, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* The same with 4-bit weights. */
int dlfp_gated_linear_w4(int32_t m, int32_t n, int32_t k, const void* x, int64_t ldx,
                         const void* gate_codes, const void* gate_exps, const void* up_codes,
                         const void* up_exps, int32_t activation, void* out, int64_t ldo,
                         int32_t out_dtype, void* workspace, size_t workspace_bytes,
                         hipStream_t stream);

/* Bytes of workspace that the fastest form of a projection takes (at most 32 MiB; 0 if it needs
 * none, and for sizes that the call refuses). */
#define DLFP_LINEAR_W4 0
#define DLFP_GATED_LINEAR_BF16 1
#define DLFP_GATED_LINEAR_W4 2
int64_t dlfp_projection_workspace(int32_t kind, int32_t m, int32_t n, int32_t k);

/* The form that a call takes with so many bytes of workspace (0: with none), rows less than 2^22
 * elements apart: for profiles and tests. */
typedef struct {
  int32_t variant;          /* its place among the kind's variants */
  int32_t rows, tokens;     /* of a workgroup's tile: rows of weights (gated: both), tokens */
  int32_t splits;           /* workgroups that share the K of a tile */
  int32_t past_caches;      /* 1: weights are read past the caches */
  int32_t reserved;
  int64_t workspace_bytes;  /* that it uses */
} dlfp_projection_form;

/* DLFP_OK, or the error of a call of these sizes (m > 0, k < 2^22), which leaves form as it is. */
int dlfp_projection_form_of(int32_t kind, int32_t m, int32_t n, int32_t k, size_t workspace_bytes,
                            dlfp_projection_form* form);

#ifdef __cplusplus
}
#endif

#endif /* DLFP_FFN_H */
