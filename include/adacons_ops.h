/*
 * adacons_ops.h -- C ABI of the training operators beside the aggregation (NVIDIA B200, sm_100a).
 *
 * The conventions are those of adacons.h: every function returns an adacons_error code, none throws
 * or aborts; pointers are device pointers unless said otherwise; `cuda_stream` is a cudaStream_t
 * passed as void*; calls are asynchronous on that stream, allocate nothing (create calls do) and
 * perform no host synchronisation; results are deterministic (no floating-point atomics, fixed
 * reduction order); no wait inside a kernel lasts longer than 2 s.
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
 *            fp16 operands with the iterate held in 22 bits; the result is within about one bf16
 *            rounding.  fp32: operands as pairs of fp16 values, about 1e-6 of the result's norm.
 *   rows, cols, offsets  host arrays; matrices must not overlap and must lie inside [0, d); sides up to 2^18.
 *            Elements outside the matrices (biases, gains) are neither read nor written.
 *   scaling  0: none; 1: each matrix's result times sqrt(max(1, rows / cols)).
 *   coeffs   host array of 3 * steps values a, b, c (one triple per step), 1 <= steps <= 64.  Iterates
 *            are held to |x| < 32; coefficients that let them grow beyond give Inf or NaN.
 *   eps      >= 0.  A matrix of zeros gives zeros when eps > 0.  Inf or NaN in a matrix give NaN in
 *            that matrix only.
 * adacons_orth_create allocates about 8 bytes per element of the matrices and 4 (bf16) or 8 (fp32) per
 * element of their short sides squared.
 * Errors: EINVAL, ELIMIT (a side beyond 2^18), ENOMEM, ECUDA, EARCH.
 */
typedef struct adacons_orth adacons_orth;

int adacons_orth_create(adacons_orth **out, int dtype, int64_t d, int num_matrices, const int64_t *rows,
                        const int64_t *cols, const int64_t *offsets, int scaling, int steps,
                        const double *coeffs, double eps);

/* One pass over the vector.  update and out may be the same buffer; any element alignment is served
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

#ifdef __cplusplus
}
#endif
#endif /* ADACONS_OPS_H_ */
