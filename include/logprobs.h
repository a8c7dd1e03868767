/*
 * libpatconv, log probabilities: what a model answers with, out of the rows of logits that its last
 * (block-pruned) product wrote, on NVIDIA B200 (sm_100a).
 *
 * For every row x[r][0..vocab-1], with lse = log sum_i exp(x_i) and p_i = exp(x_i - lse):
 *
 *   logprob[r]        = x[token[r]] - lse
 *   entropy[r]        = -sum_i p_i log p_i
 *   top[r][j]         = index of the j-th largest logit; of equal ones the lowest index comes first
 *   top_logprob[r][j] = x[top[r][j]] - lse
 *
 * A logit of -infinity is a token that may not be given: it adds nothing to lse and entropy and is never
 * among the top; where fewer than `top` others are left, the rest of top is -1 and of top_logprob -infinity.
 * A row of nothing but -infinity has an entropy of 0 and log probabilities of -infinity.  A row that holds a
 * NaN or +infinity has NaN everywhere and -1 in top.
 *
 * The row is read once; sums are fp32 (relative error of a sum about 1e-6 at most), logarithms and results fp32: off by some 1e-6, too,
 * where they are near 0.  No log probability is above 0, no entropy below.
 * Same conventions as patconv.h: plain C ABI, every function returns a status.
 */
#ifndef XGEN_LOGPROBS_H
#define XGEN_LOGPROBS_H

#include "patconv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct xgen_logprobs_packed xgen_logprobs_packed; /* opaque; holds the description */

typedef struct {
    int32_t vocab;      /* logits of a row, >= 1                                    */
    int32_t top;        /* alternatives per row, 0 .. 32, at most vocab             */
    xgen_dtype dtype;   /* of the logits: XGEN_F32 or XGEN_F16_F32ACC               */
} xgen_logprobs_desc;

/*
 * Make a handle.  device: CUDA device ordinal, or -1 for a handle that cannot run (no CUDA call is made).
 * Errors: INVALID_ARG (null pointer, vocab or top out of range), UNSUPPORTED (dtype), ALLOC, CUDA (no such device).
 */
xgen_status xgen_logprobs_pack(const xgen_logprobs_desc *desc, int device, xgen_logprobs_packed **out);

/*
 * Run over `rows` rows.
 *   x_dev           [rows] rows of vocab logits, row_stride elements apart (>= vocab), element-aligned
 *   token_dev       [rows] int32, or NULL with logprob_dev NULL.  A token of -1 asks for nothing (logprob 0);
 *                   any other that is not 0 .. vocab-1 gives NaN
 *   logprob_dev     [rows] fp32 or NULL
 *   entropy_dev     [rows] fp32 or NULL
 *   top_dev         [rows][top] int32; NULL exactly where the handle's top is 0
 *   top_logprob_dev [rows][top] fp32; likewise
 * Outputs must overlap neither the inputs nor each other.  Only enqueues one kernel on the stream, on the handle's
 * device; no workspace.  rows = 0 does nothing.
 * Errors: INVALID_ARG (null or misaligned pointer, overlap, nothing asked for), SHAPE (rows < 0 or above 2^31-1, a stride below vocab or above 2^31,
 * logits beyond 2^62 bytes), CUDA.
 */
xgen_status xgen_logprobs_run(const xgen_logprobs_packed *packed, const void *x_dev, int64_t rows, int64_t row_stride,
                              const int32_t *token_dev, float *logprob_dev, float *entropy_dev, int32_t *top_dev,
                              float *top_logprob_dev, void *cuda_stream);

/* Release the handle.  NULL is allowed. */
void xgen_logprobs_free(xgen_logprobs_packed *packed);

#ifdef __cplusplus
}
#endif
#endif /* XGEN_LOGPROBS_H */
