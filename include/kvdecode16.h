/*
 * kvdecode16.h -- C ABI of libkvdecode.so, third part: a serving step over a
 * 16-bit paged KV cache that the caller owns.  Norms and position rotation of
 * queries and keys, their write into pages, and decode attention for batches
 * whose requests share a long prefix.
 *
 * The vision tokens of a request come first in its cache (HeteroServe, Sec. 5.1,
 * the [1, N_v, d] embedding), thousands of them for an image at dynamic
 * resolution or a video; several requests may ask about the same one.  Decode
 * attention is bound by reading K and V (Sec. 2 "Language decoding"), so what
 * several rows of a batch attend to is read once for all of them here.
 *
 * The conventions of kvdecode4.h hold: everything belongs to the caller, calls
 * enqueue asynchronous work on `stream`, allocate and synchronise nothing, and
 * may be captured into CUDA graphs; lengths, ids, slots and positions are
 * device memory that is read when the kernels run; return codes come with
 * kv_last_error(), and nothing is enqueued where a call returns an error.
 * Tensors are [rows][heads][head_dim] with dense heads; "stride" is the distance
 * of two rows in elements.  Data pointers are 16-byte aligned and strides
 * multiples of 8.  What a call writes must not overlap what else it reads or
 * writes, except where it says so.  All pointers are memory of the current
 * device.  device_error (device int32, or NULL) receives KVC_DEVERR_* bits,
 * OR-ed and never cleared.  Every launch is placed while the one before it on
 * its stream finishes, and reads and writes nothing before that has completed.
 */
#ifndef KVDECODE16_H
#define KVDECODE16_H

#include <stdint.h>

#include "kvdecode4.h"

#ifdef __cplusplus
extern "C" {
#endif

/* kv16_attention: the workspace holds no plan of this batch, these heads and this head_dim. */
#define KVC_DEVERR_PLAN 16

/* A pool of one layer: K and V, each [num_pages][num_kv_heads][16 tokens][head_dim],
 * the layout that kv_cache_pool exposes; kv_tables_step hands out its pages. */
typedef struct kv16_pool {
    void *k;               /* device, 16-byte aligned                             */
    void *v;
    int64_t num_pages;     /* >= 1; num_pages * num_kv_heads < 2^27               */
    int32_t num_kv_heads;  /* 1 .. 1024                                           */
    int32_t head_dim;      /* 64 or 128                                           */
    int32_t dtype;         /* KVC_DTYPE_*: of K, V, q, out and the norms' weights */
} kv16_pool;

/* A rotation by positions.  Pair j < rotary_dim / 2 of a head's first
 * rotary_dim elements, (j, j + rotary_dim / 2) or (2 j, 2 j + 1), is turned by
 *
 *     angle = 2 pi * frac(position[axes[j]] * frequencies[j] / 2^64)
 *
 * (x, y) -> scale * (x cos - y sin, y cos + x sin); elements past rotary_dim
 * stay as they are.  The product is a whole number of 2^-64 turns, so far
 * positions lose nothing. */
typedef struct kv_rope {
    const uint64_t *frequencies; /* device [rotary_dim / 2], 8-byte aligned: turns per position, in units of 2^-64 */
    const uint8_t *axes;         /* device [rotary_dim / 2]: the axis of each pair; NULL: axis 0.
                                    A number past the last axis counts as the last one. */
    int32_t rotary_dim;          /* a multiple of 16 up to head_dim                */
    int32_t num_axes;            /* 1 .. 8: rows of positions                      */
    int32_t neighbours;          /* 0: pairs (j, j + rotary_dim / 2); 1: (2 j, 2 j + 1) */
    float scale;                 /* of cos and sin; finite                         */
} kv_rope;

/* Norms and rotation of n packed rows of queries and keys in one pass: with a
 * weight (device [head_dim], dtype), y = x / sqrt(mean(x^2) + eps) * weight over
 * each head, else y = x; then the rotation, if any.  In 32 bits, rounded once.
 *   rope       NULL: no rotation
 *   positions  device int32 [num_axes][n], rows axis_stride apart (0: all axes
 *              read the same row; negative positions turn backwards)
 *   q, q_out   device [n][num_q_heads][head_dim]; q_out may be q with the same
 *              stride.  num_q_heads 0: no queries; num_kv_heads likewise for k, k_out
 *   q_weight, k_weight  device [head_dim], 16-byte aligned; NULL: no norm
 *   eps        2^-100 .. 2^100 (looked at where there is a weight)
 * Row strides of outputs are >= heads * head_dim (n > 1), of inputs >= 0. */
KVC_API int kv_qk_rope(const kv_rope *rope, int32_t dtype, int32_t head_dim, int32_t n, const int32_t *positions,
                       int64_t axis_stride, int32_t num_q_heads, const void *q, int64_t q_stride, void *q_out,
                       int64_t q_out_stride, int32_t num_kv_heads, const void *k, int64_t k_stride, void *k_out,
                       int64_t k_out_stride, const void *q_weight, const void *k_weight, float eps, void *stream);

/* The same for n new tokens of a paged cache: normed and rotated keys, and the
 * values as they are, go to the tokens' slots (device int64 [n], page * 16 +
 * position % 16, distinct, as kv_tables_step gives them), the queries (or none:
 * num_q_heads 0) to q_out, which may be q as above.  The positions that kv_tables_step
 * gives count a request's own tokens: where it continues a prefix (kv16_plan), the
 * caller adds the first position behind that.  A slot of -1 is skipped, another one outside the pool
 * is skipped and sets KVC_DEVERR_PAGE_RANGE; the token's queries are written in
 * either case.  Without rope and weights it is a plain write. */
KVC_API int kv16_write(const kv16_pool *pool, const kv_rope *rope, int32_t n, const int64_t *slots,
                       const int32_t *positions, int64_t axis_stride, int32_t num_q_heads, const void *q,
                       int64_t q_stride, void *q_out, int64_t q_out_stride, const void *k, int64_t k_stride,
                       const void *v, int64_t v_stride, const void *q_weight, const void *k_weight, float eps,
                       int32_t *device_error, void *stream);

/* Bytes of the workspace of kv16_plan and kv16_attention for batches of up to
 * max_batch rows (<= 4096) on the current device, or a negative KVC_ERR_*. */
KVC_API int64_t kv16_workspace_bytes(const kv16_pool *pool, int32_t num_q_heads, int32_t max_batch);

/* The plan of one decode step, made on the GPU from lengths that live there,
 * for the attention of all its layers (pools of one shape).
 *   seq_ids     device [batch] (<= 4096): the request whose tokens are row r's own;
 *               NULL: row r is request r.  Requests may repeat
 *   prefix_ids  device [batch]: the request whose tokens row r attends to before
 *               its own, -1: none; NULL: none for all.  A prefix is a request of
 *               the same tables.  Rows that share one should follow one another: each
 *               run of neighbours with the same prefix reads it once.  (Keys are in the
 *               pool as they were turned: positions of own tokens behind a prefix are
 *               the caller's, see kv16_write)
 *   workspace   device, 256-byte aligned, workspace_bytes >= kv16_workspace_bytes()
 *               for this batch.  It holds this plan until the next one, and serves
 *               calls that are ordered on one stream
 * A row whose request or prefix is out of range, or has a length that is negative
 * or above max_pages * 16, sets KVC_DEVERR_SEQ_RANGE; it gets zeros and lse = -infinity.
 * Rows that together pass 2^31 pages times KV heads set the same bit, and no plan is
 * made. */
KVC_API int kv16_plan(const kv16_pool *pool, const kv_tables *tables, int32_t num_q_heads, int32_t batch,
                      const int32_t *seq_ids, const int32_t *prefix_ids, void *workspace, int64_t workspace_bytes,
                      int32_t *device_error, void *stream);

/* Decode attention of the planned rows, one token each:
 * o = sum_t softmax_t(softmax_scale q . k_t) v_t over the tokens of the row's prefix
 * and its own, whose numbers are those that kv16_plan found and whose pages are
 * read from the block tables now.
 *   q, out   device [batch][num_q_heads][head_dim], row strides q_stride (>= 0) and
 *            out_stride; num_q_heads / num_kv_heads <= 8
 *   lse      device [batch][num_q_heads] float, out, or NULL: the natural
 *            logarithm of each softmax's denominator, sum_t exp(scale q.k_t)
 * softmax_scale (below 2^100) <= 0 selects 1 / sqrt(head_dim).  A row without
 * tokens gives zeros and lse = -infinity.  The tokens of a page id outside the
 * pool are left out, with KVC_DEVERR_PAGE_RANGE.  A workspace without a plan
 * of this batch, num_q_heads and pool shape sets KVC_DEVERR_PLAN, and nothing is
 * written.  Waits in the kernel end after a second or so: should one run out, the call and
 * those that follow by the same plan set KVC_DEVERR_WAIT_TIMEOUT, and outputs are NaN.  Scores, softmax statistics and sums are held in 32 bits: scores of any
 * size that are numbers there give weights that are.  Weights
 * meet V in the pool's type, at most half a step of it off (fp16: weights below 2^-21 of the
 * largest, 2^-32 of that).  Outputs that would round to an infinity are the type's
 * largest number; sums of weights up to 2^8 times V have to be numbers of 32 bits (bf16:
 * V below 2^88 always is).  The result of a call
 * does not depend on timing: partial results are merged in a fixed order. */
KVC_API int kv16_attention(const kv16_pool *pool, const kv_tables *tables, int32_t batch, int32_t num_q_heads,
                           const void *q, int64_t q_stride, void *out, int64_t out_stride, float *lse,
                           float softmax_scale, void *workspace, int64_t workspace_bytes, int32_t *device_error,
                           void *stream);

#ifdef __cplusplus
}
#endif

#endif /* KVDECODE16_H */
