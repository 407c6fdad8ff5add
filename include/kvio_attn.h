/*
 * kvio_attn.h -- what a model does with the paged cache that kvio.h moves, on
 * the same pool handles: kvio_append writes new tokens' keys and values into
 * their sequences' pages (rotating keys and queries by their positions on the
 * way), kvio_attend computes causal attention of new tokens over those pages.
 *
 * The cache holds 16-bit elements (bf16, fp16) or e4m3 codes with one fp32
 * scale for each (pool page, KV head) of K and of V: an element's value is its
 * code times the scale of its page and head.  The scales of a layer are two
 * device arrays, [num_pages][scale_stride] each (H used of every row), that
 * the caller owns and passes with each call; a pool of elem_bytes 4, head_dim
 * 1 and page size 1 over them moves them between host and GPU beside the codes
 * (H * 4 must then be a multiple of 16).
 *
 * Conventions are kvio.h's: kvio_status, kvio_last_error, asynchronous on the
 * given stream, arguments checked before anything is enqueued, nothing
 * allocated and no memset (so the calls can be captured into a HIP graph),
 * every buffer the caller's.  The lengths, offsets and page tables of a batch
 * are read on the GPU when the call runs: a replayed graph follows their values of
 * then.  All pointers are device memory of the pool's GPU, which has to be the
 * current device.
 */
#ifndef KVIO_ATTN_H
#define KVIO_ATTN_H

#include "kvio.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define KVIO_BF16 0
#define KVIO_FP16 1
#define KVIO_E4M3 2       /* 8 bits: 4 of exponent, 3 of mantissa, largest 448, no infinity */

/* New tokens of several sequences, one row each in the call's q, k, v, out.
 * Sequence b has rows [q_start[b], q_start[b + 1]), the last of the ctx_len[b]
 * tokens of its context: row q_start[b + 1] - 1 - j is context token
 * ctx_len[b] - 1 - j.  Context token t lives in pool slot
 * page_table[b][t / P] * P + t % P.
 * Values that make no sense are cut to what is there: offsets to [0,
 * num_tokens], lengths to [0, max_pages * P], new tokens
 * to the first max_query.  Offsets must not fall: a sequence that ends before it begins has no rows, and it is not
 * defined which of the rows that the others name are worked on then, nor for which; no other rows or pages are
 * touched.  A row whose place comes out below zero, or whose page lies
 * outside the pool, is not appended; a cached token whose page lies outside the
 * pool is attended by nobody.  The first such page is reported by kvio_check
 * (span = the sequence). */
typedef struct kvio_batch {
    int32_t num_seqs;           /* B >= 0                                                    */
    int32_t num_tokens;         /* N >= 0 rows that the arrays of new tokens hold            */
    int32_t max_pages;          /* entries of one sequence in page_table, >= 1               */
    int32_t max_query;          /* most new tokens of any sequence; 0 = num_tokens           */
    int64_t table_stride;       /* entries from one sequence's to the next's, >= max_pages   */
    const int32_t *page_table;  /* int32[B][table_stride]                                    */
    const int32_t *ctx_len;     /* int32[B]                                                  */
    const int32_t *q_start;     /* int32[B + 1]; NULL: one new token each, row b (N >= B)    */
} kvio_batch;

/* Write the batch's new tokens into layer `layer` of the pool.
 * Rotation (rot_dim > 0) turns pair i of the first rot_dim elements of every
 * head of K and Q by the angle position * inv_freq[i], the product taken in 64
 * bits: (a, b) becomes (a cos - b sin, b cos + a sin).  The position is the token's place in its
 * context, or positions[row].  Pair i is elements (i, i + rot_dim / 2), or
 * with KVIO_APPEND_INTERLEAVED (2i, 2i + 1).  The result is rounded once to `dtype`.
 * In e4m3 a page's scale of a head is the smallest power of two 2^e, e >= -100,
 * with all elements that the page has taken since its first token within 448 * 2^e: a page whose
 * first token is among the new ones starts anew, one that is filled further
 * keeps its scale unless new elements pass 448 times it, or it is (from elsewhere) below 2^-100 in size,
 * infinite or NaN; then its rows are rounded again under the new one (exact but for codes below the smallest
 * normal one, where both are powers of two).  Elements are rounded to nearest even; infinities
 * become +-448 times the scale and do not raise it, NaN stays NaN.
 * No two rows of a call may name one pool slot, in e4m3 no two sequences one page
 * that they append to.  Rows of no sequence are left alone, in q_out too. */
#define KVIO_APPEND_INTERLEAVED 0x1
typedef struct kvio_append_args {
    kvio_batch batch;
    int32_t dtype;              /* of q, k, v, q_out: KVIO_BF16 or KVIO_FP16                 */
    int32_t cache_dtype;        /* of the pool: `dtype` itself or KVIO_E4M3                  */
    int32_t num_q_heads;        /* heads of q; 0 without q                                   */
    int32_t rot_dim;            /* elements of a head that are rotated, a multiple of 16, <= D; 0 = none */
    int32_t flags;              /* KVIO_APPEND_*                                             */
    int32_t reserved;           /* 0                                                         */
    const void *k, *v;          /* [N][H][D], tokens k_stride / v_stride elements apart      */
    const void *q;              /* [N][num_q_heads][D] or NULL                               */
    void *q_out;                /* where rotated q goes: q itself, or memory apart from it (slices of one */
                                /*   buffer's rows are, where the strides are equal)         */
    int64_t k_stride, v_stride, q_stride, q_out_stride;  /* multiples of 8                   */
    const float *inv_freq;      /* fp32[rot_dim / 2]                                         */
    const int32_t *positions;   /* int32[N] or NULL                                          */
    float *k_scale, *v_scale;   /* e4m3: the layer's scales                                  */
    int64_t scale_stride;       /* floats from one page's to the next's, >= H                */
} kvio_append_args;

/* D a multiple of 16 up to 1024; q, k, v and q_out 16-byte aligned. */
kvio_status kvio_append(kvio_pool_t pool, int32_t layer, const kvio_append_args *args, hipStream_t stream);

/* Attention of the batch's new tokens over their contexts in layer `layer`:
 *   out[row][h] = sum over t of softmax_t(softmax_scale * q[row][h] . K[t][g]) * V[t][g],
 * g = h / (num_q_heads / H), t over the context tokens up to the row's own and, with
 * window > 0, the last `window` of those only.  A row that sees no token gets zeros and an lse
 * of minus infinity; lse[row][h] (if not NULL) is the natural logarithm of the softmax's sum.
 * What hidden tokens hold, infinities and NaN included, has no effect, nor have scales, such ones included, of pages that
 * a row sees no token of (but for the precision that is named below).
 * Products are accumulated in fp32, probabilities rounded to 16 bits for the second one: to the cache's type (fp16 in
 * steps of 2^-31 of the row's largest at least), with an e4m3 cache to fp16, times their values' scales (a scale below 2^-18 of the context's largest, tokens that the row does
 * not see included, loses precision).  With up to 64 rows to a KV head (max_query times query heads; 32 with D of 256) what
 * that takes off is added as a second term (not for bf16 queries over e4m3, whose results do not show it).
 * Equal inputs give equal bits, except over other max_pages, max_query or GPUs.
 * Rows of no sequence are left alone. */
typedef struct kvio_attend_args {
    kvio_batch batch;
    int32_t dtype;              /* of q and out: KVIO_BF16 or KVIO_FP16                      */
    int32_t cache_dtype;        /* of the pool: `dtype` itself or KVIO_E4M3                  */
    int32_t num_q_heads;        /* a multiple of the pool's H                                */
    int32_t window;             /* 0 = none                                                  */
    float softmax_scale;        /* > 0, and finite times log2(e)                             */
    int32_t reserved;           /* 0                                                         */
    const void *q;              /* [N][num_q_heads][D], tokens q_stride elements apart       */
    void *out;                  /* [N][num_q_heads][D], out_stride apart                     */
    float *lse;                 /* fp32[N][num_q_heads] or NULL                              */
    int64_t q_stride, out_stride;  /* multiples of 8                                         */
    const float *k_scale, *v_scale;  /* e4m3: the layer's scales                             */
    int64_t scale_stride;
    void *workspace;            /* kvio_attend_workspace bytes, 16-byte aligned; contents    */
    size_t workspace_bytes;     /*   need not survive between calls, overlapping calls need their own */
} kvio_attend_args;

/* D of 64, 128 or 256; q and out 16-byte aligned, memory apart from each other (as q and q_out above). */
kvio_status kvio_attend(kvio_pool_t pool, int32_t layer, const kvio_attend_args *args, hipStream_t stream);

/* Bytes of workspace that kvio_attend takes for these arguments; follows from the batch's sizes and
 * types (not from pointers, which may be NULL here) and may be 0. */
kvio_status kvio_attend_workspace(kvio_pool_t pool, const kvio_attend_args *args, size_t *bytes);

#ifdef __cplusplus
}
#endif

#endif /* KVIO_ATTN_H */
