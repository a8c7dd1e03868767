/*
 * libpatconv, low-rank adapters: what many requests, each with an adapter of its own, add to a product that
 * they share (a block-pruned one of blockgemm.h, say), on NVIDIA B200 (sm_100a).
 *
 * An adapter a is a pair of matrices A_a [rank][k] and B_a [c_out][rank] and a scale s_a.  The rows of x are
 * grouped by request: request i owns the rows row_start[i] .. row_start[i+1]-1 and has the adapter
 * adapter[i], or none (a negative number).  For every such row r and output channel oc
 *
 *   out[r][oc] = y[r][oc] + s_a * sum_j B_a[oc][j] * (sum_c A_a[j][c] * x[r][c])
 *
 * and out[r] = y[r] where the request has no adapter.  Both sums are fp32; the inner one is kept to 11 bits relative to its row's
 * largest in fp16 layers, the result is rounded once.  fp32 layers keep fp32's precision throughout (relative error of
 * a sum of magnitudes about 1e-6).  A row of x, or an adapter, with values that are not finite gives results that are not
 * finite (a NaN where the sums would be infinite, too) in the rows that use it, and in no others.
 *
 * Same conventions as patconv.h: plain C ABI, every function returns a status, *_host is host memory, *_dev
 * memory of the device the handle was packed for.
 */
#ifndef XGEN_ADAPTERS_H
#define XGEN_ADAPTERS_H

#include "patconv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct xgen_adapters_packed xgen_adapters_packed; /* opaque; owns device memory */

typedef struct {
    int32_t k;           /* input features, >= 1                                             */
    int32_t c_out;       /* output channels, >= 1                                            */
    int32_t rank;        /* columns of B, rows of A: 1 .. 128 (adapters of a lower rank are padded with zeros) */
    int32_t adapters;    /* how many, >= 1                                                    */
    xgen_dtype dtype;    /* XGEN_F32, or XGEN_F16_F32ACC (x, A, B, y, out IEEE fp16)          */
} xgen_adapters_desc;

/*
 * Lay out and upload a set of adapters.
 *   a_host      [adapters][rank][k] in the dtype's element type (fp16 as IEEE bits)
 *   b_host      [adapters][c_out][rank] likewise
 *   scale_host  [adapters] fp32
 *   device      CUDA device ordinal, or -1 for a handle that cannot run (no CUDA call is made)
 * Synchronous; inputs are copied.  Errors: INVALID_ARG, UNSUPPORTED (dtype, rank), SHAPE (k or c_out above 2^24, or more
 * than 2^40 bytes), ALLOC, CUDA.
 */
xgen_status xgen_adapters_pack(const xgen_adapters_desc *desc, const void *a_host, const void *b_host, const float *scale_host, int device,
                               xgen_adapters_packed **out);

/*
 * Run over `rows` rows of `requests` requests.
 *   x_dev         [rows] rows of k elements, x_stride elements apart
 *   row_start_dev [requests+1] int32, not falling, within 0 .. rows
 *   adapter_dev   [requests] int32: 0 .. adapters-1, or negative for none
 *   y_dev         [rows] rows of c_out elements, y_stride apart
 *   out_dev       [rows] rows of c_out elements, out_stride apart: y_dev itself with the same stride (in place), or
 *                 memory that does not overlap y_dev; never memory of x_dev
 * Pointers element-aligned; rows that all start on a multiple of 16 bytes are moved 16 bytes at a time.  Rows that no request owns are
 * neither read nor written.  Row numbers outside 0 .. rows are cut to that range; an adapter number too high
 * counts as none and, where its request has rows, is reported by xgen_adapters_last_status.
 * Only enqueues one kernel on the stream, on the handle's device; no workspace.  rows = 0 or requests = 0 does nothing.
 * Errors: INVALID_ARG (null or misaligned pointer, overlap), SHAPE (negative sizes, a stride below the
 * row's length or above 2^31, rows or requests above 2^31-1, too many of both for one launch), CUDA.
 */
xgen_status xgen_adapters_run(const xgen_adapters_packed *packed, const void *x_dev, int64_t rows, int64_t x_stride,
                              const int32_t *row_start_dev, const int32_t *adapter_dev, int64_t requests, const void *y_dev,
                              int64_t y_stride, void *out_dev, int64_t out_stride, void *cuda_stream);

/* Synchronise the stream and report the first error seen: XGEN_OK, XGEN_ERR_CUDA, or, once, XGEN_ERR_INVALID_ARG
 * after a run that met an adapter number that is too high. */
xgen_status xgen_adapters_last_status(const xgen_adapters_packed *packed, void *cuda_stream);

/* Release the handle and its device memory.  NULL is allowed. */
void xgen_adapters_free(xgen_adapters_packed *packed);

#ifdef __cplusplus
}
#endif
#endif /* XGEN_ADAPTERS_H */
