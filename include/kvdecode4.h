/*
 * kvdecode4.h -- C ABI of libkvdecode.so, second part: a paged KV cache held
 * in 4 bits, single-token decode attention that reads it, and the block tables
 * and slot maps of a serving step built on the GPU from request lengths.
 *
 * A decode step streams the K and V of every cached token from HBM
 * (HeteroServe, Sec. 2 "Language decoding"), 2 * L * n_kv * d_h * s_ctx * b
 * bytes a request (Sec. 4.1, Eq. 1): b = 2 for the cache of kvdecode.h, 0.53 to
 * 0.63 here.  Attention is that of decode_attention (kvdecode.h) with every K
 * and V element replaced by the value that its code stands for.
 *
 * Everything belongs to the caller and is passed in: pools, tables, maps and
 * workspace.  The conventions of kvdecode.h hold: return codes with
 * kv_last_error(), asynchronous work on `stream`, no call synchronises or
 * allocates, and nothing is enqueued where a call returns an error.  All calls
 * may be captured into CUDA graphs: lengths, ids and slots are device memory
 * and are read when the kernels run.  Tensors are row-major; "stride" is the
 * distance of two tokens' (or two requests') rows in elements, the heads of a
 * row are dense: [rows][heads][head_dim].  Data pointers are 16-byte aligned
 * and their strides multiples of 8 elements; what a call writes must not
 * overlap what else it reads or writes.  device_error (device int32, or NULL)
 * receives KVC_DEVERR_* bits, OR-ed and never cleared.
 *
 * Every launch is placed while the one before it on its stream finishes
 * (programmatic dependent launch) and reads and writes nothing before that
 * has completed.
 */
#ifndef KVDECODE4_H
#define KVDECODE4_H

#include <stdint.h>

#include "kvdecode.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KVC_DTYPE_BF16 0
#define KVC_DTYPE_F16 1

/* A pool of one layer: num_pages pages of 16 tokens of num_kv_heads KV heads,
 * [num_pages][num_kv_heads] blocks of
 *
 *     K codes  [16 * head_dim / 2 bytes]
 *     V codes  [16 * head_dim / 2 bytes]
 *     K scales [16 tokens][head_dim / group] words
 *     V scales [16 tokens][head_dim / group] words
 *
 * A scale word holds s in its low and z in its high 16 bits, both in the
 * pool's dtype, for `group` consecutive elements of one token; a code c in
 * 0 .. 15 stands for s * (c - 8) + z.  Codes are 32-bit words of eight:
 *
 *     K word [token][j][i], j < 4, i < head_dim / 32: element d = 32 i + 8 j + e,
 *       e < 8, in bits 16 (e % 2) + 4 (e / 2) and up;
 *     V word [token / 8][g][j][i], g < 8, j < 4: token 8 (token / 8) + 2 j + h and
 *       element d = 32 i + 8 n + g, h < 2, n < 4, in bits 16 h + 4 n and up.
 *
 * Quantisation of a group's values x: s = rn16((max/2 - min/2) / 7.5),
 * z = rn16(min + 8 s), c = clamp(rint((x - z) / s) + 8, 0, 15), with the
 * difference and the sum in 32 bits, rn16 and rint (of the exact quotient) to
 * nearest even; c = 8 where s is 0.  Where z + 7 s or z - 8 s would round to an
 * infinity (a group that holds numbers at the end of the type's range), s is the next
 * smaller number and z = min + 8 s is rounded toward zero: what is finite stays finite.
 * A group that holds an infinity or a NaN stands for NaN in all its elements. */
typedef struct kv4_pool {
    void *data;            /* device, kv4_pool_bytes() bytes, 128-byte aligned   */
    int64_t num_pages;     /* 1 .. 2^31 - 1                                      */
    int32_t num_kv_heads;  /* 1 .. 1024                                          */
    int32_t head_dim;      /* 64 or 128                                          */
    int32_t group;         /* elements that share a scale: 32, 64 or head_dim    */
    int32_t dtype;         /* KVC_DTYPE_*: of q, k, v, out, and of s and z       */
} kv4_pool;

/* Block tables of up to max_seqs requests.  Request i holds lens[i] tokens on
 * the pages block_table[i][0 .. ceil(lens[i] / 16) - 1]; entries past those
 * hold anything.  The free pages are free_ring[(free_state[0] + k) %
 * num_pages], k < free_state[1], the next one to be handed out first;
 * free_state[2] and [3] belong to the library and start at zero.  A request's
 * pages are its own.  They serve the pools of this header: decode_attention_noalloc takes its
 * lengths from the host.  Tokens given back are drafts that the caller has rejected; what
 * verifies them lies with the caller, the attention here takes one token a request. */
typedef struct kv_tables {
    int32_t *block_table;  /* device, [max_seqs][max_pages]                      */
    int32_t *lens;         /* device, [max_seqs]                                 */
    int32_t *free_ring;    /* device, [num_pages]; NULL where only read          */
    int32_t *free_state;   /* device, [4]: first, number of free pages, 0, 0     */
    int64_t num_pages;     /* entries of free_ring; page ids are below it        */
    int32_t max_seqs;
    int32_t max_pages;     /* max_seqs * max_pages < 2^31                        */
} kv_tables;

/* Bytes of a pool (data is not looked at), or a negative KVC_ERR_*. */
KVC_API int64_t kv4_pool_bytes(const kv4_pool *pool);

/* One step's block tables and slot map for `batch` distinct requests
 * (batch <= 4096), from their lengths on the device (the pages of a request
 * are taken when it needs them: Sec. 5.4 "Lazy KV Cache Allocation"; the new
 * tokens of all requests are one packed batch: Sec. 5.4 "Flash Attention
 * Varlen for Packed Prefill").
 *   seq_ids   device [batch]: request of each batch row; NULL: row i is request i
 *   new_lens  device [batch]: n > 0 adds n tokens, -n gives the last n back
 *             (rejected draft tokens; all of them: the request is closed)
 *   slots     device [max_tokens] int64, out: page * 16 + position % 16 of every
 *             new token, requests in batch order; -1 past the last one and for
 *             tokens of a refused request
 *   positions device [max_tokens] int32, out, or NULL: positions of the same, -1 as above
 *   cu_seqlens device [batch + 1] int32, out, or NULL: first new token of each
 *             row (rows that give back count 0), then their number
 *   lens_out  device [max_seqs] int32, out: all lengths after the step; NULL: in place
 *   free_state_out  device [4], out ([0] and [1] are written); NULL: in place
 * Pages are taken from the ring in batch order and written into the block
 * table; pages given back go to the ring's end, in batch order and a
 * request's pages in logical order, and are handed out from the next call on.
 * A request is refused, its length and tables kept, where its row would
 * pass max_pages or a length fall below zero or its id is out of range
 * (KVC_DEVERR_SEQ_RANGE), where its new tokens pass max_tokens (the same), or
 * where the free pages do not cover what it and the rows before it need
 * (KVC_DEVERR_OOM; rows that need no page still grow).  A page id outside the
 * pool sets KVC_DEVERR_PAGE_RANGE; its tokens get slot -1, and where it is given back it is
 * left out: it does not become a free page.  Should the
 * pages given back not fit the ring (a page given back twice), all rows that
 * give back are refused with KVC_DEVERR_PAGE_RANGE. */
KVC_API int kv_tables_step(const kv_tables *tables, int32_t batch, const int32_t *seq_ids, const int32_t *new_lens,
                           int32_t max_tokens, int64_t *slots, int32_t *positions, int32_t *cu_seqlens,
                           int32_t *lens_out, int32_t *free_state_out, int32_t *device_error, void *stream);

/* Quantise the K and V rows of n tokens (k, v: device [n][num_kv_heads]
 * [head_dim], row strides k_stride, v_stride >= 0) into their slots (device [n],
 * as kv_tables_step gives them; distinct).  A slot of -1 is skipped, another
 * one outside the pool is skipped and sets KVC_DEVERR_PAGE_RANGE. */
KVC_API int kv4_write(const kv4_pool *pool, int32_t n, const int64_t *slots, const void *k, int64_t k_stride,
                      const void *v, int64_t v_stride, int32_t *device_error, void *stream);

/* The values of n tokens' slots (any order, repeats allowed), rounded to the
 * pool's dtype, into k_out and v_out (device [n][num_kv_heads][head_dim], row
 * strides >= num_kv_heads * head_dim).  Rows of slot -1 become zero; so do
 * those of a slot outside the pool, which sets KVC_DEVERR_PAGE_RANGE. */
KVC_API int kv4_read(const kv4_pool *pool, int32_t n, const int64_t *slots, void *k_out, int64_t k_stride,
                     void *v_out, int64_t v_stride, int32_t *device_error, void *stream);

/* Bytes of kv4_decode_attention's workspace on the current device, or a
 * negative KVC_ERR_*: the same for every batch and length.  What it holds
 * between calls does not matter; it serves calls that are ordered on one stream. */
KVC_API int64_t kv4_workspace_bytes(const kv4_pool *pool, int32_t num_q_heads);

/* Decode attention of `batch` rows (<= 4096) over all lens[i] tokens of each
 * row's request i = seq_ids[row] (device [batch], or NULL: i = row); requests may repeat.
 *   q, out    device [batch][num_q_heads][head_dim], row strides q_stride (>= 0) and
 *             out_stride (>= num_q_heads * head_dim); num_q_heads / num_kv_heads <= 8
 *   lse       device [batch][num_q_heads] float, out, or NULL: the natural
 *             logarithm of each softmax's denominator, sum_t exp(scale q.k_t)
 *   workspace device, workspace_bytes >= kv4_workspace_bytes(), 256-byte aligned
 * softmax_scale (below 2^100) <= 0 selects 1 / sqrt(head_dim).  A request of length 0 gives
 * zeros and lse = -infinity; so does one whose id is out of range or whose length is
 * negative or above max_pages * 16, with KVC_DEVERR_SEQ_RANGE.  The tokens of a
 * page id outside the pool are left out, with KVC_DEVERR_PAGE_RANGE.  Rows that
 * together pass 2^31 pages times KV heads set KVC_DEVERR_SEQ_RANGE and nothing
 * is written.  Scores, softmax statistics and sums are held in 32 bits.  What meets
 * V's codes, a token's weight times its scale, is rounded to 11 bits, below 2^-20 of the
 * largest of its sum (a query head's over the elements of a scale group) to
 * multiples of 2^-30 of that.  Outputs that would round to an infinity are the type's
 * largest number; sums of weights up to 16 times V have to be numbers of 32 bits (bf16: V
 * below 2^90 always is).  A q that is not finite gives NaN.  The result of a call does
 * not depend on timing: partial results are merged in the order of their tokens. */
KVC_API int kv4_decode_attention(const kv4_pool *pool, const kv_tables *tables, int32_t batch, const int32_t *seq_ids,
                                 int32_t num_q_heads, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                                 float *lse, float softmax_scale, void *workspace, int64_t workspace_bytes,
                                 int32_t *device_error, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* KVDECODE4_H */
