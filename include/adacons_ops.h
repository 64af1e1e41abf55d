/*
 * adacons_ops.h -- C ABI of the training operators beside the aggregation (NVIDIA B200, sm_100a).
 *
 * The conventions are those of adacons.h: every function returns an adacons_error code, none throws
 * or aborts; pointers are device pointers unless said otherwise, of the device that was current when the
 * context was created, whichever is current at the call (attention has no context: of the device that is
 * current); `cuda_stream` is a cudaStream_t of that device passed as void*; calls are asynchronous on that
 * stream, allocate nothing (create calls do) and perform no host synchronisation; results are deterministic
 * (no floating-point atomics, fixed reduction order); no wait inside a kernel lasts longer than 2 s.
 */
#ifndef ADACONS_OPS_H_
#define ADACONS_OPS_H_

#include "adacons.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------------
 * Orthogonalisation of an update, matrix by matrix, by Newton-Schulz products.
 *
 * A flat vector of d elements (the aggregated direction, or an optimiser's momentum of it) holds
 * num_matrices row-major matrices, rows[k] x cols[k] at element offsets[k].  Each one is replaced by
 *     X = G / (|G|_F + eps);   steps times:  X <- a X + (b S + c S S) X,  S = X X^T;   out = scale X
 * taken on its short side.  With the usual coefficients (3.4445, -4.7750, 2.0315) five steps bring
 * all singular values that are not tiny near one.
 *   dtype    ADACONS_F32 or ADACONS_BF16: storage of the update and of the result.  bf16: products of
 *            fp16 operands with the iterate held in 22 bits; the result is within 2.4e-3 of its norm (one bf16
 *            rounding is 1.7e-3), 4e-3 where all singular values are alike, 1.6e-2 on sides below 16.
 *            fp32: operands as pairs of fp16 values, about 1e-6 of the result's norm.
 *   rows, cols, offsets  host arrays; matrices must not overlap and must lie inside [0, d); sides up to 2^18.
 *            Elements outside the matrices (biases, gains) are neither read nor written.
 *   scaling  0: none; 1: each matrix's result times sqrt(max(1, rows / cols)).
 *   coeffs   host array of 3 * steps values a, b, c (one triple per step), 1 <= steps <= 64.  What the steps hold in 16-bit
 *            parts must stay in their range: elements of X below 32, of S = X X^T below 8 (no row of X longer than
 *            2.8, as no singular value beyond that), of a I + b S + c S S below 32.  Coefficients that let
 *            them grow beyond give Inf or NaN; the usual ones stay below 1.3, 1.5 and 3.5.
 *   eps      >= 0.  A matrix of zeros gives zeros when eps > 0.  Inf or NaN in a matrix give NaN in
 *            that matrix only.
 * adacons_orth_create allocates about 8 bytes per element of the matrices and 4 (bf16) or 8 (fp32) per
 * element of their short sides squared; up to 19 MB more for a matrix whose long rows are split between blocks.
 * Errors: EINVAL, ELIMIT (a side beyond 2^18), ENOMEM, ECUDA, EARCH.
 */
typedef struct adacons_orth adacons_orth;

int adacons_orth_create(adacons_orth **out, int dtype, int64_t d, int num_matrices, const int64_t *rows,
                        const int64_t *cols, const int64_t *offsets, int scaling, int steps,
                        const double *coeffs, double eps);

/* One pass over the vector.  update and out may be the same buffer, otherwise they must not overlap; any element alignment is served
 * (16-byte aligned buffers, offsets and rows that are multiples of 8 elements let the result be written in vectors).  A context holds the iterates:
 * calls on one context must be ordered (one stream, or events).  Errors: EINVAL, ECUDA. */
int adacons_orth_apply(adacons_orth *ctx, const void *update, void *out, void *cuda_stream);

/* ADACONS_FLAG_TIMEOUT if a bounded wait expired since the last call (the results since are invalid);
 * clears it.  Synchronises `cuda_stream`. */
int adacons_orth_get_status(adacons_orth *ctx, uint32_t *flags, void *cuda_stream);

enum adacons_orth_info {
  ADACONS_ORTH_INFO_BYTES = 0,    /* device bytes owned by the context */
  ADACONS_ORTH_INFO_LAUNCHES = 1  /* kernels launched by the most recent adacons_orth_apply */
};
int adacons_orth_get_info(adacons_orth *ctx, int key, int64_t *value);

/* The caller makes sure that no work of the context is still running.  NULL is accepted. */
int adacons_orth_destroy(adacons_orth *ctx);

/* ------------------------------------------------------------------------------------------------
 * Attention and its gradient.
 *
 * Per query head:  S = scale Q K^T, -inf where a query does not see a key;  lse = log sum exp S;
 *     O = exp(S - lse) V
 * Key j is visible to query i when j < kv_lens[batch] and, with `causal`, j <= i + kv_len - q_len (the
 * last query sees the last key).  A query that sees no key has O = 0, lse = -inf, and takes no part in any
 * gradient, whatever its q and dO hold.  Keys from kv_lens[batch] on may hold anything, Inf and NaN included; their gradients are 0.
 * Query heads h kv_heads / q_heads share a key head; its gradients are the sums over them.
 */
enum { ADACONS_F16 = 2 }; /* attention takes ADACONS_BF16 and ADACONS_F16 */

/* A tensor of 16-bit elements (batch, token, head, element): strides in elements, the last one is 1.
 * Any order of the first three dimensions is served (slices of a packed projection, head-major or
 * token-major).  data must be 16-byte aligned, and the strides positive multiples of 8; those of
 * dimensions of size 1 are not looked at. */
typedef struct adacons_attn_tensor {
  void *data;
  int64_t batch_stride, seq_stride, head_stride;
} adacons_attn_tensor;

typedef struct adacons_attn_shape {
  int dtype;              /* ADACONS_BF16 or ADACONS_F16 */
  int batch;              /* 0 .. 65535 */
  int q_heads, kv_heads;  /* q_heads a multiple of kv_heads */
  int q_len, kv_len;      /* tokens, 0 .. 2^30 */
  int head_dim;           /* a multiple of 8 up to 128 */
  int causal;             /* 0 or 1 */
  float scale;            /* > 0; usually head_dim^-1/2 */
  const int32_t *kv_lens; /* device pointer, `batch` values (clamped to 0 .. kv_len), or NULL: all keys */
} adacons_attn_shape;

/* out: as q; lse: (batch, q_heads, q_len) fp32, contiguous.  out must not overlap the inputs (EINVAL where it starts with k or v).
 * Errors: EINVAL, EALIGN, ELIMIT (head_dim > 128, sizes beyond the above), ECUDA, EARCH. */
int adacons_attn_forward(const adacons_attn_shape *shape, const adacons_attn_tensor *q, const adacons_attn_tensor *k,
                         const adacons_attn_tensor *v, const adacons_attn_tensor *out, float *lse, void *cuda_stream);

/* dq, dk, dv from dout, with the probabilities recomputed from lse.  dq, dk and dv are written, not added to,
 * and must not overlap the inputs or one another (EINVAL where two start together).  workspace: device memory of adacons_attn_workspace_bytes, 16-byte
 * aligned, free for other use after the call's work.  It may be NULL where q_heads / kv_heads times q_len, rounded
 * up to a multiple of 128, is at most ADACONS_ATTN_SHORT_ROWS (fp16: and kv_len at most ADACONS_ATTN_SHORT_KEYS): one
 * launch instead of two, each block making for itself what the first would leave there; quicker for a few short heads.
 * Probabilities and dS are operands of the products in the tensors' type.  fp16 holds them scaled by powers of two (dS from the
 * largest norms of dout's and v's rows), so that neither long rows nor small or large dout leave its range.
 * Errors: as the forward pass. */
#define ADACONS_ATTN_SHORT_ROWS 256
#define ADACONS_ATTN_SHORT_KEYS 4096
int adacons_attn_workspace_bytes(const adacons_attn_shape *shape, int64_t *bytes);
int adacons_attn_backward(const adacons_attn_shape *shape, const adacons_attn_tensor *dout, const adacons_attn_tensor *q,
                          const adacons_attn_tensor *k, const adacons_attn_tensor *v, const adacons_attn_tensor *out,
                          const float *lse, const adacons_attn_tensor *dq, const adacons_attn_tensor *dk,
                          const adacons_attn_tensor *dv, void *workspace, int64_t workspace_bytes, void *cuda_stream);

/* ADACONS_FLAG_TIMEOUT if a bounded wait expired in an attention kernel of the current device since the last
 * call (results since are invalid); clears it.  Synchronises `cuda_stream`. */
int adacons_attn_get_status(uint32_t *flags, void *cuda_stream);

/* ------------------------------------------------------------------------------------------------
 * Rotary positions.
 *
 * Pair i of a head at position t is turned by the angle t f_i and multiplied by `gain`:
 *     (a, b) -> gain (a cos - b sin, a sin + b cos)
 * with (a, b) = elements (i, i + rot/2) of the head or, interleaved, (2i, 2i+1).  Elements from `rot` on
 * pass through unchanged.  The gradient of the turn is the turn by the negative angle with the same gain:
 * inverse = 1.
 *   rot          even, 2 .. 4096: the rotated elements of a head.
 *   frequencies  host array of rot/2 angles per position, in radians; any scaling for long contexts is in
 *                them.  The angle is formed and reduced in fp64: positions up to 2^31 keep their precision.
 * Errors: EINVAL, ELIMIT, ENOMEM, ECUDA, EARCH.
 */
typedef struct adacons_rope adacons_rope;
int adacons_rope_create(adacons_rope **out, int rot, const double *frequencies, double gain, int interleaved);

typedef struct adacons_rope_shape {
  int dtype;                 /* ADACONS_F32 or ADACONS_BF16 */
  int batch, len, heads;     /* heads * head_dim up to 2^26 */
  int head_dim;              /* >= rot */
} adacons_rope_shape;

/* x, y: (batch, token, head, element) with the element stride 1; x_strides, y_strides: host arrays of the
 * other three strides in elements, any values.  y may be x with the same strides, otherwise they must not overlap.
 * positions: device pointer to batch * len values in that order (contiguous), or NULL: token s of every
 * sequence is at position first + s.  16-byte aligned data whose strides and rot, head_dim are multiples of
 * 16 bytes (rot of 32) are moved in vectors, anything else element by element.  Errors: EINVAL, ELIMIT, ECUDA. */
int adacons_rope_apply(adacons_rope *ctx, const adacons_rope_shape *shape, const void *x, const int64_t *x_strides, void *y,
                       const int64_t *y_strides, const int32_t *positions, int64_t first, int inverse, void *cuda_stream);

/* NULL is accepted. */
int adacons_rope_destroy(adacons_rope *ctx);

/* ------------------------------------------------------------------------------------------------
 * Self-tests of the hang protection, as adacons_selftest_bounded_wait: the kernels of a call with one tile left
 * out, so that the waits behind it run out after 2 s each, the blocks let go of what they hold and return, and the
 * status word says ADACONS_FLAG_TIMEOUT.  The results are invalid, the next call's are not touched by it.
 *   adacons_selftest_orth       adacons_orth_apply whose first tile nobody computes; EINVAL for a context all of whose
 *                               matrices fit one block (128 x 256), whose kernel has no such wait
 *   adacons_selftest_attention  the forward pass (dq NULL) or the gradient, with out in the place of dout; every block
 *                               lacks its last tile.  ADACONS_BF16 and head_dim up to 64, otherwise EINVAL
 */
int adacons_selftest_orth(adacons_orth *ctx, const void *update, void *out, void *cuda_stream);
int adacons_selftest_attention(const adacons_attn_shape *shape, const adacons_attn_tensor *q, const adacons_attn_tensor *k,
                               const adacons_attn_tensor *v, const adacons_attn_tensor *out, float *lse, const adacons_attn_tensor *dq,
                               const adacons_attn_tensor *dk, const adacons_attn_tensor *dv, void *workspace, int64_t workspace_bytes, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* ADACONS_OPS_H_ */
