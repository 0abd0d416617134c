/*
 * hs_kv8.h -- rotary positions and the 8-bit cache of the full-attention layers (hs_attn.h has the
 * 16-bit cache and hs_attn_shape, hs.h the conventions shared by every call).
 *
 *   hs_rope_plan            the angles of a model's positions (host)
 *   hs_rope_apply           q and k turned by their positions
 *   hs_kv8_append           new tokens' K and V rows quantised into their 8-bit pages
 *   hs_kv8_append_rope      hs_rope_apply and hs_kv8_append in one launch
 *   hs_kv8_decode           one decode step of a batch over the 8-bit pages
 *   hs_kv8_read             a prefix read back into 16-bit pages, for hs_attn_prefill
 */
#ifndef HS_KV8_H
#define HS_KV8_H

#include "hs_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Tokens that share a scale. */
#define HS_KV8_GROUP 16

/* Which elements of a head make the pair i < dims / 2. */
typedef enum hs_rope_layout {
    HS_ROPE_HALF = 0,        /* i and i + dims / 2 */
    HS_ROPE_INTERLEAVED = 1  /* 2 i and 2 i + 1 */
} hs_rope_layout;

/* How positions are scaled for contexts longer than the trained one (hs_rope_plan). */
typedef enum hs_rope_scaling {
    HS_ROPE_PLAIN = 0,   /* not at all */
    HS_ROPE_LINEAR = 1,  /* every angle divided by the factor */
    HS_ROPE_BASE = 2,    /* a larger base: base * factor^(dims / (dims - 2)) */
    HS_ROPE_TURNS = 3,   /* slow pairs divided by the factor, the share between linear in a pair's turns */
    HS_ROPE_INDEX = 4    /* the same with the share linear in the pair's index */
} hs_rope_scaling;

#define HS_ROPE_MAX_PAIRS 64

/* A model's positions, filled in by hs_rope_plan (or by the caller, for other angles).  Passed by address,
 * read by the host before a call returns. */
typedef struct hs_rope {
    int32_t dims;       /* the first dims elements of a head are turned; a multiple of 16, at most head_dim */
    int32_t layout;     /* hs_rope_layout */
    double amplitude;   /* factor of the turned elements, 2^-20 to 2^20 (1: lengths are kept) */
    double theta[HS_ROPE_MAX_PAIRS]; /* angle of pair i for each position, in radians; below 2^64 in magnitude */
} hs_rope;

/*
 * hs_rope_plan -- the angles of rotary positions (host only, no GPU).
 *
 * With theta_i = base^(-2 i / dims) and t_i = context * theta_i / (2 pi), the turns that pair i makes
 * over the trained context:
 *     HS_ROPE_PLAIN    theta_i
 *     HS_ROPE_LINEAR   theta_i / factor
 *     HS_ROPE_BASE     (base * factor^(dims / (dims - 2)))^(-2 i / dims)
 *     HS_ROPE_TURNS    theta_i (s + (1 - s) / factor),  s = (t_i - low) / (high - low) cut to [0, 1]
 *     HS_ROPE_INDEX    the same with s = 1 - (i - a) / (b - a) cut to [0, 1], where
 *                      x(t) = dims ln(context / (2 pi t)) / (2 ln base) is the index of the pair that makes
 *                      t turns, a = max(floor(x(high)), 0), b = min(ceil(x(low)), dims - 1), and b - a is at
 *                      least 0.001
 *   dims       a multiple of 16, 16 to 128
 *   layout     hs_rope_layout
 *   base       > 1 and finite
 *   scaling    hs_rope_scaling
 *   factor     >= 1 and finite (HS_ROPE_PLAIN ignores it)
 *   context    tokens that the unscaled positions were trained for, >= 1 (TURNS and INDEX alone)
 *   low, high  turns, 0 < low < high, finite (TURNS and INDEX alone)
 *   amplitude  2^-20 to 2^20
 * Errors: HS_ERR_INVALID_ARG, HS_ERR_UNSUPPORTED (dims).
 */
hs_status hs_rope_plan(int32_t dims, int32_t layout, double base, int32_t scaling, double factor,
                       int64_t context, double low, double high, double amplitude, hs_rope *out);

/*
 * hs_rope_apply -- the rows of q and k turned by their positions.
 *
 * Paper: Section 2.2 (the suffix [B,N) continues at its absolute positions, so that its rows meet the
 * restored ones as in the recomputation).
 *
 * For row r, every head and pair (x, y) of it, with c = cos(pos[r] theta_i), s = sin(pos[r] theta_i):
 *     x' = amplitude (x c - y s),   y' = amplitude (y c + x s)
 * Elements from rope->dims on are copied.
 *   shp        n_heads, n_kv_heads, head_dim and dtype are used
 *   q, k       device, row r at element r * in_stride: [n_heads][head_dim], [n_kv_heads][head_dim]; views into
 *              a fused projection's output are fine.  Either may be NULL: its rows are left out
 *   in_stride  elements between rows of both, a multiple of 8; 0: q's n_heads * head_dim, k's
 *              n_kv_heads * head_dim
 *   pos        device int64 [n_rows]; negative positions turn backwards.  theta is rounded to a multiple of 2^-64
 *              turns and the angle reduced exactly, so that it is off by |pos| 2^-65 turns at most (1.5e-9 radians at
 *              2^33) beside float32's roundings
 *   q_out, q_out_stride, k_out, k_out_stride  device, the results, laid out alike (a stride of 0: the rows touch).
 *              In place is fine: q_out == q with the same stride, k_out == k with the same stride.  They must
 *              not overlap otherwise
 * Arithmetic: sine and cosine, products and sums in float32, rounded once to the element type.
 * Pointers 16-byte aligned (pos: 8).
 * Errors: HS_ERR_INVALID_ARG, HS_ERR_MISALIGNED, HS_ERR_UNSUPPORTED (head_dim, n_kv_heads > 1024,
 * n_heads / n_kv_heads > 128, 2^31 rows), HS_ERR_CUDA.
 */
hs_status hs_rope_apply(const hs_attn_shape *shp, const hs_rope *rope, const void *q, const void *k,
                        int64_t in_stride, const int64_t *pos, int64_t n_rows, void *q_out,
                        int64_t q_out_stride, void *k_out, int64_t k_out_stride, cudaStream_t stream);

/*
 * The 8-bit cache of a layer: num_blocks blocks of hs_kv8_block_bytes bytes, each
 *     [n_kv_heads][2][page_size][head_dim] E4M3 (plane 0 the keys, plane 1 the values), then
 *     [n_kv_heads][2][page_size / 16] float scales, padded to a multiple of 128 bytes.
 * A value is its E4M3 number times the scale of its KV head, plane and group of 16 tokens; scales are powers of
 * two from 2^-126 to 2^120.  A block is a page that hs_restore_kv_pages, hs_restore_request and
 * hs_save_kv_pages move (page_bytes = the block's bytes): its scales travel with it.  Key j of a request lies
 * in block block_table[request][j / page_size] as token j % page_size.
 * KV heads h to h + n - 1 of a block are two ranges, the values and behind all values the scales.
 * hs_restore_kv_page_slices and hs_save_kv_page_slices move each with rows = 1:
 *     values  col_off = h * B,                   col_bytes = n * B,  B = 2 * page_size * head_dim
 *     scales  col_off = n_kv_heads * B + h * S,  col_bytes = n * S,  S = page_size / 2
 * which have to be multiples of 16: with pages of 16 tokens h and n are even.
 *
 * shp->dtype is the type of q, k, v, o and of the 16-bit cache, not of this one's.
 */

/* The bytes of one block: n_kv_heads * 2 * (page_size * head_dim + page_size / 16 * 4), rounded up to 128. */
hs_status hs_kv8_block_bytes(const hs_attn_shape *shp, int64_t *bytes_out);

/*
 * hs_kv8_append -- quantise new tokens' K and V rows of one layer into the 8-bit cache.
 *
 * Paper: Table 1 (the FP8 KV setting), Section 2.2 and Section 5.5, as hs_kv_append.
 *
 * Arguments, slots and skipped rows as hs_kv_append.  Of every group of 16 tokens that gets rows, KV head and
 * plane, with M the largest magnitude among the new values and need = the smallest 2^e >= M / 448, e >= -126:
 *   - a group whose first token (slot % 16 == 0) is among the rows is begun anew: its scale becomes need,
 *     its other tokens' bytes stay as they are (and mean nothing until they are written);
 *   - another goes on: its scale becomes the larger of the one it has and need, and where it grows, what the
 *     group's other tokens hold is rounded to it.
 * New values are divided by the scale and rounded to the nearest E4M3 number (ties to even).  So a value is
 * off by at most 2^-4 of itself, or by 2^-10 of the scale where that is more, and once more for each time that its
 * group's scale grew: at most 16 times in all, since a group has 16 tokens.
 * The rows of a group must stand within 16 rows (in any order), with none but skipped rows among them, as the new tokens of
 * a request do, and slots >= 0 must be distinct: else the group's values mean nothing.  A value that is not finite becomes
 * NaN and takes no part in M.
 * k, v and the cache must be 16-byte aligned and must not overlap.
 * Errors: as hs_kv_append (HS_ERR_UNSUPPORTED also for 2^31 rows).
 */
hs_status hs_kv8_append(const hs_attn_shape *shp, const void *k, const void *v, int64_t kv_stride,
                        const int64_t *slots, int64_t n_rows, void *cache, int32_t *d_err,
                        cudaStream_t stream);

/*
 * hs_kv8_append_rope -- hs_rope_apply of q into q_out and hs_kv8_append of the turned k, and of v, in one
 * launch.
 *
 * k's turned values are not rounded to the element type in between: at positions below 2^39 in magnitude scales and bytes
 * are those of the exactly turned keys (what float32 leaves open is decided with twice its bits).  Where a
 * turned value is beyond float32's range, both of its pair count as not finite; where amplitude times an element is, they
 * may.  Rows with a negative slot
 * are skipped altogether: their row of q_out is not written.  A row whose slot is out of range is turned into q_out.
 *   in_stride  elements between rows of q, k and v, a multiple of 8; 0: each one's own heads * head_dim
 *   q_out      as hs_rope_apply (in place is fine); q and q_out may both be NULL
 * Everything else, and the errors: as hs_rope_apply and hs_kv8_append.
 */
hs_status hs_kv8_append_rope(const hs_attn_shape *shp, const hs_rope *rope, const void *q, const void *k,
                             const void *v, int64_t in_stride, const int64_t *pos, const int64_t *slots,
                             int64_t n_rows, void *q_out, int64_t q_out_stride, void *cache,
                             int32_t *d_err, cudaStream_t stream);

/*
 * hs_kv8_decode -- hs_attn_decode over an 8-bit cache.
 *
 * Paper: Table 1 (the FP8 KV setting), Section 5.1 and Section 5.5 (128-token continuations after the resume).
 *
 * Arguments and results as hs_attn_decode, with K and V the cache's values.
 * Arithmetic: q . k as products of binary16 numbers with float32 sums (E4M3 fits it; a bf16 q is scaled by a
 * power of two for each row, elements below 2^-24 of its largest lose bits and those below 2^-39 count as zero);
 * maxima, sums and lse in float32; the weights times the values' scales as the sum of two binary16 numbers before the
 * product with v (2^-22 relative, or 2^-32 of the row's largest weight times the largest scale where that is more); the
 * outputs once at the end, kept within the element type's finite values.
 * Scores must lie within float32's range; a weight below 2^-126 of the row's largest counts as zero.
 * With shp->unsplit a row's result depends on nothing but its query and its keys; without it, the keys of one
 * row may be shared out by the sizes of the call, and equal calls give equal bits.
 * Nothing of the cache at or behind kv_len[b] reaches a result, whatever it holds.  Where a key or value in front of it is
 * NaN, that request's outputs of the KV head's heads need not be finite; the others keep their values.
 *   block_table  an id outside [0,num_blocks) sets HS_DEVERR_BLOCK_OOB; its page is not read, and the outputs
 *                of that request mean nothing
 * HS_DEVERR_TIMEOUT from this call: none of its outputs means anything.  Its waits are bounded by 1 s.
 * Errors: as hs_attn_decode (HS_ERR_UNSUPPORTED also for more than 2^31 groups of 16 tokens in all, with every
 * request at max_kv_len, and for a cache of 2^38 bytes or more).
 */
hs_status hs_kv8_decode(const hs_attn_shape *shp, const void *q, const void *cache,
                        const int32_t *block_table, const int32_t *kv_len, int64_t max_kv_len, void *o,
                        float *lse, void *workspace, int64_t workspace_bytes, int32_t *d_err,
                        cudaStream_t stream);

/* The workspace hs_kv8_decode needs for this shape and bound (with the current device). */
hs_status hs_kv8_decode_workspace_bytes(const hs_attn_shape *shp, int64_t max_kv_len, int64_t *bytes_out);

/*
 * hs_kv8_read -- the first kv_len[b] tokens of each request read back into 16-bit pages.
 *
 * Paper: Section 2.2 (the restored entries of [0,B) are attended to by the recomputed suffix).
 *
 * For key j < kv_len[b]: block out_table[b][j / page_size] of `out`, a cache as in hs_attn.h with out_blocks
 * blocks, gets the values of the 8-bit cache's key j, rounded to the element type (exact but below fp16's normal
 * numbers; kept within the type's finite values).  Other tokens of the pages are not written.
 *   shp        batch, n_kv_heads, head_dim, page_size, dtype, num_blocks, max_pages are used
 *   block_table, out_table  device int32 [batch][max_pages], of request b the first
 *              ceil(kv_len[b] / page_size) entries are read.  An id outside [0,num_blocks) or
 *              [0,out_blocks) sets HS_DEVERR_BLOCK_OOB, and that page is skipped
 *   kv_len     device int32 [batch], 0 <= kv_len[b] <= max_kv_len (else HS_DEVERR_LENGTH, and the request is
 *              skipped)
 *   max_kv_len host, 0 to max_pages * page_size
 * The listed pages of `out` must be distinct where both requests write to them with different values.  cache and out
 * 16-byte aligned, not overlapping.
 * Errors: HS_ERR_INVALID_ARG, HS_ERR_MISALIGNED, HS_ERR_UNSUPPORTED (as hs_kv_append, batch > HS_MAX_BATCH,
 * max_kv_len near 2^31), HS_ERR_CUDA.
 */
hs_status hs_kv8_read(const hs_attn_shape *shp, const void *cache, const int32_t *block_table,
                      const int32_t *kv_len, int64_t max_kv_len, void *out, int64_t out_blocks,
                      const int32_t *out_table, int32_t *d_err, cudaStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* HS_KV8_H */
