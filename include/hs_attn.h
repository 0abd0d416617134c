/*
 * hs_attn.h -- the full-attention layers of a resumed request (hs.h has the rest, and the
 * conventions shared by every call).
 *
 * For each full-attention layer, over the pages that hs_restore_kv_pages restored:
 *   hs_kv_append            write the tail's (or the step's) new K and V rows into their pages
 *   hs_attn_prefill         causal attention of the tails [c,N) of a batch
 *   hs_attn_decode          one decode step of a batch
 *   hs_attn_decode_shared   one decode step of requests behind one cached prefix
 */
#ifndef HS_ATTN_H
#define HS_ATTN_H

#include "hs.h"

#ifdef __cplusplus
extern "C" {
#endif

/* one more code that a kernel may store into d_err */
#define HS_DEVERR_LENGTH 5        /* a length read from a device array is < 0 or above the call's bound */
/* HS_DEVERR_TIMEOUT from an attention call: none of its outputs means anything.  Its waits are bounded by 1 s and
 * 20 us for each tile of 128 keys that one CTA may have to walk. */

/* Element type of the attention calls' q, o and cache. */
typedef enum hs_dtype {
    HS_BF16 = 0, /* bfloat16 */
    HS_FP16 = 1  /* IEEE binary16 */
} hs_dtype;

/* One full-attention layer of a batch of requests (the attention calls and hs_kv_append).
 *
 * Cache of the layer: [num_blocks][2][page_size][n_kv_heads][head_dim], plane 0 the keys, plane 1
 * the values, so that a block is one of the pages that the restore and save calls move
 * (page_bytes = 2 * page_size * n_kv_heads * head_dim * 2).  Key j of a request lies in block
 * block_table[request][j / page_size] at row j % page_size.
 *
 * Query head h reads KV head h / (n_heads / n_kv_heads). */
typedef struct hs_attn_shape {
    int32_t batch;         /* requests, 0 to HS_MAX_BATCH (hs_kv_append ignores it) */
    int32_t n_heads;       /* query heads; a multiple of n_kv_heads, at most 128 times it */
    int32_t n_kv_heads;
    int32_t head_dim;      /* 64 or 128 */
    int32_t page_size;     /* tokens per page: 16, 32, 64, 128 or 256 */
    int32_t dtype;         /* hs_dtype */
    int64_t num_blocks;    /* blocks of the cache */
    int64_t max_pages;     /* entries in each row of block_table */
    int64_t q_stride;      /* elements between rows of q, a multiple of 8; 0: n_heads * head_dim */
    int64_t o_stride;      /* the same of o */
    float scale;           /* factor of q . k, > 0 and finite (usually head_dim^-1/2) */
    int32_t unsplit;       /* 1: the keys of one row are never shared out over CTAs (see
                              hs_attn_prefill); 0: as is fastest */
} hs_attn_shape;

/*
 * hs_kv_append -- write new tokens' K and V rows of one layer into the paged cache.
 *
 * Paper: Section 2.2 (the suffix [B,N) is recomputed, so its attention entries are written
 * anew) and Section 5.5 (128-token continuations extend the cache token by token).
 *
 * For row r < n_rows with slots[r] >= 0, b = slots[r] / page_size, i = slots[r] % page_size:
 *     cache[b][0][i][:][:] <- k[r],   cache[b][1][i][:][:] <- v[r]
 * Rows with a negative slot (padding) are skipped; one at or above num_blocks * page_size sets
 * HS_DEVERR_BLOCK_OOB and is skipped.  Slots >= 0 must be distinct (two equal ones race).
 *   shp        n_kv_heads, head_dim, page_size, dtype and num_blocks are used
 *   k, v       device, row r at element r * kv_stride: [n_kv_heads][head_dim]; views into a
 *              fused projection's output are fine
 *   kv_stride  elements between rows, a multiple of 8; 0: n_kv_heads * head_dim
 *   slots      device int64 [n_rows]
 *   cache      device, the layer's cache
 * k, v and the cache must be 16-byte aligned and must not overlap.
 * Errors: HS_ERR_INVALID_ARG, HS_ERR_MISALIGNED, HS_ERR_UNSUPPORTED (head_dim, page_size, n_kv_heads > 1024,
 * 2^31 8-token groups in the cache), HS_ERR_CUDA.
 */
hs_status hs_kv_append(const hs_attn_shape *shp, const void *k, const void *v, int64_t kv_stride,
                       const int64_t *slots, int64_t n_rows, void *cache, int32_t *d_err,
                       cudaStream_t stream);

/*
 * hs_attn_prefill -- causal attention of a batch of tails over their paged keys.
 *
 * Paper: Section 2.1 and Section 2.2 (a resumed request continues over [B,N) with the attention
 * entries of [0,B) restored; B = 0 is the recomputation).
 *
 * Token t < n_tokens[b] of request b is row cu_rows[b] + t of q and o and absolute position
 * p = pos0[b] + t.  Per head, over the keys of its KV head,
 *     o_t = sum_{j <= p} w_j v_j,   w_j = exp(scale q_t.k_j - lse_t),
 *     lse_t = log sum_{j <= p} exp(scale q_t.k_j)
 * The keys of positions [0, pos0 + n_tokens) must be in the cache (hs_restore_kv_pages,
 * hs_kv_append); nothing of the cache at later positions reaches a result, whatever it holds.
 *   shp          host
 *   q            device, row r at element r * q_stride: [n_heads][head_dim]
 *   cache        device, the layer's cache
 *   block_table  device int32 [batch][max_pages]; of request b the first
 *                ceil((pos0 + n_tokens) / page_size) entries are read (none if it has no tokens).
 *                Requests may share blocks.  An id outside [0,num_blocks) sets
 *                HS_DEVERR_BLOCK_OOB; the outputs of the rows that attend to that page then mean
 *                nothing (the page is not read)
 *   o            device, row r at element r * o_stride: [n_heads][head_dim]; rows of no token are
 *                not written
 *   lse          device float [rows][n_heads] (natural logarithm), or NULL
 *   pos0, n_tokens  host int64 [batch], int32 [batch]; pos0 + n_tokens <= max_pages * page_size
 *   cu_rows      host int64 [batch + 1], as in hs_linattn_prefill_packed
 *   workspace    device, 16-byte aligned, at least hs_attn_prefill_workspace_bytes bytes (NULL
 *                where that is 0); contents on entry ignored, on return undefined.  Calls that can
 *                run at the same time need workspaces of their own
 * Arithmetic: products of q and k and of the weights and v on 16-bit operands with float32 sums;
 * maxima, sums and lse in float32; the weights rounded to the element type (2^-8 relative for
 * bf16; 2^-11 for fp16, or half a step of 2^-32 of the row's largest weight where that is more) before the
 * product with v, the outputs once at the end.
 * The tensor core adds to a float32 sum and drops what lies below 2^-26 of it: where one CTA walks n keys
 * (`unsplit`, or a row of a long prefill) and a column's values are of one sign, an output is low by up to
 * n 2^-27 of it (8e-4 at 131,072 keys; measured).
 * Scores may lie anywhere in float32's range; each is good to some 2^-24 of the sum of its products' magnitudes, so
 * that of scores of 10^7 and more only ones that lie well apart are told apart.
 * With shp->unsplit a row's result depends on nothing but its query and its keys, so a tail resumed
 * at any position equals the recomputation bit for bit; without it, the keys of one row may be
 * shared out over CTAs by the sizes of the call, and equal calls give equal bits.
 * K and V of the positions below pos0 + n_tokens should be finite.  Where one in v_j is not, the
 * outputs of the positions p >= j are not finite in its column (NaN possibly in place of an
 * infinity); where one in k_j is not, none of those positions' outputs need be.  Earlier positions and
 * other requests keep their values.
 * All pointers 16-byte aligned; o and lse must not overlap anything else.
 * Errors: HS_ERR_INVALID_ARG, HS_ERR_MISALIGNED, HS_ERR_UNSUPPORTED (head_dim, page_size,
 * n_heads / n_kv_heads > 128, n_kv_heads > 1024, batch > HS_MAX_BATCH, a stride, position, row times heads or
 * number of 8-token groups in the cache near 2^31 or above, 2^31 tiles of 128 keys in all), HS_ERR_CUDA.
 */
hs_status hs_attn_prefill(const hs_attn_shape *shp, const void *q, const void *cache,
                          const int32_t *block_table, void *o, float *lse, const int64_t *pos0,
                          const int32_t *n_tokens, const int64_t *cu_rows, void *workspace,
                          int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream);

/* The workspace hs_attn_prefill needs for these arguments (with the current device). */
hs_status hs_attn_prefill_workspace_bytes(const hs_attn_shape *shp, const int64_t *pos0,
                                          const int32_t *n_tokens, int64_t *bytes_out);

/*
 * hs_attn_decode -- one decode step: attention of one token of each request over its keys.
 *
 * Paper: Section 5.1 and Section 5.5 (128-token continuations after the resume).
 *
 * Row b of q and o is request b's token; it attends to the kv_len[b] keys of its pages, its own
 * among them (append it first).  kv_len[b] == 0 writes o = 0 and lse = -infinity.  Lengths are
 * read on the device, so a captured step can be replayed as they grow.
 *   q, cache, block_table, o, lse, workspace, arithmetic: as hs_attn_prefill, with rows 0 to
 *                batch - 1; of request b the first ceil(kv_len[b] / page_size) entries of the
 *                table are read
 *   kv_len       device int32 [batch], 0 <= kv_len[b] <= max_kv_len (else HS_DEVERR_LENGTH, and
 *                nothing is written for that request)
 *   max_kv_len   host, 0 to max_pages * page_size; a bound of at most 384 saves the join's launch (1 us)
 * Errors: as hs_attn_prefill.
 */
hs_status hs_attn_decode(const hs_attn_shape *shp, const void *q, const void *cache,
                         const int32_t *block_table, const int32_t *kv_len, int64_t max_kv_len,
                         void *o, float *lse, void *workspace, int64_t workspace_bytes,
                         int32_t *d_err, cudaStream_t stream);

/* The workspace hs_attn_decode needs for this shape and bound (with the current device). */
hs_status hs_attn_decode_workspace_bytes(const hs_attn_shape *shp, int64_t max_kv_len,
                                         int64_t *bytes_out);

/*
 * hs_attn_decode_shared -- hs_attn_decode for requests whose prompts share a cached prefix.
 *
 * Paper: Section 2.1 (the cached entries of a prefix serve every request that begins with it).
 *
 * Each request's keys are the prefix_len keys of prefix_table's pages followed by the kv_len[b]
 * keys of its own pages in block_table (its row of the table begins with the first page behind
 * the prefix).  The prefix is read once for all requests' queries instead of once for each.  The
 * prefix may end inside a page; rows with no key at all get o = 0 and lse = -infinity.
 *   prefix_table  device int32 [ceil(prefix_len / page_size)], NULL allowed when prefix_len == 0
 *   prefix_len    host, >= 0
 *   kv_len, max_kv_len  of the keys behind the prefix
 * Everything else, and the errors: as hs_attn_decode (prefix_len + max_kv_len below 2^31).
 */
hs_status hs_attn_decode_shared(const hs_attn_shape *shp, const void *q, const void *cache,
                                const int32_t *prefix_table, int64_t prefix_len,
                                const int32_t *block_table, const int32_t *kv_len,
                                int64_t max_kv_len, void *o, float *lse, void *workspace,
                                int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream);

/* The workspace hs_attn_decode_shared needs for this shape and these bounds (with the current
 * device). */
hs_status hs_attn_decode_shared_workspace_bytes(const hs_attn_shape *shp, int64_t prefix_len,
                                                int64_t max_kv_len, int64_t *bytes_out);

#ifdef __cplusplus
}
#endif

#endif /* HS_ATTN_H */
