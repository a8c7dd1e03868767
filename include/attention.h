/*
 * libpatconv, attention over a paged cache of 8 bits: what stands between the (block-pruned) products of a
 * transformer layer when it answers, on NVIDIA B200 (sm_100a).
 *
 * A batch is a number of sequences.  Sequence i has length[i] tokens so far, of which the last ones are new in
 * this call: the rows row_start[i] .. row_start[i+1]-1 of the new keys, values or queries, at the positions length[i] - n
 * .. length[i] - 1.  (Rows whose position would be negative are neither appended nor read back, and see nothing as queries.)
 * Lengths are at most 2^30, rows at most 2^31 elements apart.
 *
 * The cache is a set of pages.  A page holds, for every key/value head, page_tokens tokens of head_dim signed
 * 8-bit codes, and one fp32 scale for the keys and one for the values: a code c stands for c * scale.
 *
 *   k_codes, v_codes  [pages][kv_heads][page_tokens][head_dim] int8
 *   k_scale, v_scale  [pages][kv_heads] fp32
 *   page_table        [sequences] rows of table_stride int32: token j of sequence i is in page
 *                     page_table[i][j / page_tokens], in slot j % page_tokens
 *
 * Rotation: component pair u of a head (components u and u + rotary/2, or 2u and 2u + 1 where interleaved, u <
 * rotary/2) at position p is turned by the angle p * freq[u]:  (a, b) -> (a cos - b sin, a sin + b cos).  Keys are stored
 * turned; queries are turned on the way in.  Components from `rotary` on stay.
 *
 * Appending to a page (per head; keys and values alike), amax = the largest magnitude of the new entries:
 *   * where the call writes slot 0, or where the page's scale is 0, the scale becomes amax/127;
 *   * otherwise the old scale s is doubled until amax <= 127.5 s, and the older codes of the page are halved as
 *     often, rounded to nearest even.  An entry is then off by less than one step of the page's scale, however often
 *     the page was appended to (the half steps of its roundings are halved each time).
 *   * code = entry / scale rounded to nearest, halves to even, within -127 .. 127.
 * A new entry that is not finite makes the page's scale NaN, and it stays NaN until slot 0 is written again: whoever
 * attends to the page (in that head) gets NaN.  Slots behind the sequence's last token are left as they were.
 *
 * Attention: query head h uses key/value head h / (q_heads/kv_heads).  The row at position p sees the tokens j <= p,
 * with a window only j > p - window.
 *   y = sum_j softmax_j( softmax_scale * <turned q, k_j> ) v_j
 * A row that sees nothing gives zeros.  Maxima and sums are fp32.  A turned query row becomes integers of 16 bits (fp32
 * layers: 24) times its largest magnitude / 32512 (8323072); their products with the codes are exact (fp16 layers,
 * sequences of many rows: kept to 23 bits).  What is added
 * up is the product of a token's probability and its value scale: it has 11 bits down to 2^-20 of the row's largest one so far (fp32 layers:
 * 22 bits down to 2^-8), and is off by 2^-31 of that largest one at most below.  Pages that the row does not see have no part in it.  A
 * probability of less than 2^-100 of the row's largest may count as none.
 *
 * Pages outside 0 .. pages-1 (or beyond table_stride) are not touched: appending to one is left out, its
 * tokens are seen by nobody and read as zeros, and xgen_attention_last_status reports it.  A page that is appended to belongs to one
 * sequence alone; pages that are only read may be shared.
 *
 * Same conventions as patconv.h: plain C ABI, every function returns a status, *_host is host memory, *_dev
 * memory of the device the handle was packed for.
 */
#ifndef XGEN_ATTENTION_H
#define XGEN_ATTENTION_H

#include "patconv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct xgen_attention_packed xgen_attention_packed; /* opaque; owns device memory */

typedef struct {
    int32_t q_heads;        /* a multiple of kv_heads                                        */
    int32_t kv_heads;       /* >= 1                                                           */
    int32_t head_dim;       /* 32, 64, 96, 128, 192 or 256                                    */
    int32_t page_tokens;    /* 16, 32, 64 or 128                                              */
    xgen_dtype dtype;       /* of queries, new keys and values, results: XGEN_F32 or XGEN_F16_F32ACC */
    int32_t rotary;         /* components turned, even, 0 .. head_dim                         */
    int32_t interleaved;    /* 0: pairs (u, u + rotary/2); 1: pairs (2u, 2u+1)                */
    int32_t window;         /* tokens that a row sees, itself among them; 0 = all before it  */
    float softmax_scale;    /* > 0, or 0 for 1/sqrt(head_dim)                                 */
} xgen_attention_desc;

typedef struct {
    int32_t sequences;              /* >= 0                                                    */
    int32_t longest;                /* at least the rows of every sequence (any bound will do; a tight one launches less).
                                       What a sequence has beyond it may be left out, which xgen_attention_last_status reports */
    int64_t rows;                   /* rows of the tensors that belong to the batch; others are left alone */
    const int32_t *row_start_dev;   /* [sequences+1], not falling, within 0 .. rows           */
    const int32_t *length_dev;      /* [sequences], the new rows included                      */
    const int32_t *page_table_dev;  /* [sequences][table_stride]                               */
    int64_t table_stride;
} xgen_attention_batch;

typedef struct {
    void *k_codes_dev, *v_codes_dev;     /* 16-byte aligned                                    */
    float *k_scale_dev, *v_scale_dev;
    int64_t pages;
} xgen_attention_cache;

/*
 * Make a handle.
 *   freq_host  [rotary/2] fp64, radians per position; NULL where rotary is 0.  (Kept as 64-bit fractions of a turn:
 *              an angle is off by some 2^-25 of a turn, at any position.)
 *   device     CUDA device ordinal, or -1 for a handle that cannot run (no CUDA call is made)
 * Errors: INVALID_ARG, UNSUPPORTED (dtype, head_dim, page_tokens, rotary), SHAPE (more than 65535 heads), ALLOC, CUDA.
 */
xgen_status xgen_attention_pack(const xgen_attention_desc *desc, const double *freq_host, int device, xgen_attention_packed **out);

/*
 * Write the batch's new keys and values into the cache.
 *   k_dev, v_dev  [rows] rows of kv_heads * head_dim elements, kv_stride elements apart (both may be parts of one
 *                 product's rows), element-aligned, outside the cache
 * Only enqueues one kernel.  Errors: INVALID_ARG (null or misaligned pointer; keys, values or what describes the batch in the cache, or its
 * parts over each other), SHAPE, CUDA.
 */
xgen_status xgen_attention_append(const xgen_attention_packed *packed, const void *k_dev, const void *v_dev, int64_t kv_stride,
                                  const xgen_attention_batch *batch, const xgen_attention_cache *cache, void *cuda_stream);

/*
 * Give back what the cache holds of the batch's rows (to hand a prefix on, to check): codes times scales, keys turned.
 *   out_dtype            XGEN_F32 or XGEN_F16_F32ACC, whatever the handle's type
 *   k_out_dev, v_out_dev [rows] rows of kv_heads * head_dim elements, out_stride apart, element-aligned, outside the cache and what describes
 *                        the batch; no element of one is one of the other's (they may be parts of the same rows)
 * Only enqueues one kernel.  Errors as for append, and UNSUPPORTED (out_dtype).
 */
xgen_status xgen_attention_read(const xgen_attention_packed *packed, const xgen_attention_batch *batch, const xgen_attention_cache *cache,
                                xgen_dtype out_dtype, void *k_out_dev, void *v_out_dev, int64_t out_stride, void *cuda_stream);

/* Bytes of workspace that xgen_attention_run takes for this batch's sequences, rows and longest (the device pointers
 * are not looked at).  It grows with rows and longest, so what does for a batch does for every smaller one.  Errors: INVALID_ARG, SHAPE, CUDA (host-only handle). */
xgen_status xgen_attention_workspace(const xgen_attention_packed *packed, const xgen_attention_batch *batch, int64_t *bytes);

/*
 * Attention of the batch's rows over the cache (which holds them already: append first).
 *   q_dev  [rows] rows of q_heads * head_dim elements, q_stride apart, element-aligned
 *   y_dev  [rows] rows likewise, y_stride apart, outside q_dev, the cache and what describes the batch
 *   workspace_dev  xgen_attention_workspace bytes, 16-byte aligned, outside all of these.  Nothing in it counts between calls; calls that
 *          may run at the same time need one each
 * Only enqueues kernels: two for a few rows of each sequence, three more where a sequence may have many.
 * Errors: INVALID_ARG (null or misaligned pointer, overlap), SHAPE (rows times q_heads / kv_heads above 2^31 - 257 too), CUDA.
 */
xgen_status xgen_attention_run(const xgen_attention_packed *packed, const void *q_dev, int64_t q_stride, const xgen_attention_batch *batch,
                               const xgen_attention_cache *cache, void *y_dev, int64_t y_stride, void *workspace_dev, void *cuda_stream);

/* Synchronise the stream and report the first error seen: XGEN_OK, XGEN_ERR_CUDA, or, once, XGEN_ERR_INVALID_ARG
 * after a call that met a page that is not there or a sequence longer than it said, or XGEN_ERR_TIMEOUT after one in which
 * a kernel's own waits ran out (two seconds; its results are not complete). */
xgen_status xgen_attention_last_status(const xgen_attention_packed *packed, void *cuda_stream);

/*
 * Testing aid, not for production use: with extra > 0 the products of every later xgen_attention_run that has many rows wait, 50 ms at
 * most, for `extra` arrivals (1000 at most) more than will ever come, so that the call ends with XGEN_ERR_TIMEOUT in
 * xgen_attention_last_status; 0 restores normal operation.  Errors: INVALID_ARG.
 */
xgen_status xgen_attention_test_expect_arrivals(xgen_attention_packed *packed, int32_t extra);

/* Release the handle and its device memory.  NULL is allowed. */
void xgen_attention_free(xgen_attention_packed *packed);

#ifdef __cplusplus
}
#endif
#endif /* XGEN_ATTENTION_H */
