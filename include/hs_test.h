/*
 * hs_test.h -- fault-injection entry points for the failure-detection tests.
 * They are not part of the restore-and-resume path and no product code calls them.
 *
 * hs_test_prefill_stalled takes the arguments of hs_linattn_prefill_from_state
 * (hs.h) and requires shp->kernel == HS_LINATTN_CHUNKED_TC (else
 * HS_ERR_UNSUPPORTED).  Every CTA of the tensor-core kernel first waits on an
 * mbarrier that nothing completes.  That wait is bounded like every wait of the
 * kernel (1 s of the GPU's global timer); when it runs out the CTA takes its
 * abort path: it stores HS_DEVERR_TIMEOUT into d_err (if d_err still holds 0),
 * waits (bounded) for its own copies in flight, frees its tensor memory and
 * returns without writing o, state or any checkpoint slot.  The context stays
 * usable, and later calls on the stream run normally.
 *
 * Argument checks, layouts, ownership and host-side errors are those of
 * hs_linattn_prefill_from_state.
 */
#ifndef HS_TEST_H
#define HS_TEST_H

#include "hs.h"
#include "hs_attn.h"
#include "hs_kv8.h"

#ifdef __cplusplus
extern "C" {
#endif

hs_status hs_test_prefill_stalled(const hs_linattn_shape *shp, const uint16_t *q, const uint16_t *k,
                                  const uint16_t *v, const float *log_g, float *o, float *state,
                                  const int64_t *pos0, const int32_t *n_tokens,
                                  int32_t ckpt_interval, float *const *ckpt_slots, int32_t *d_err,
                                  cudaStream_t stream);

/*
 * hs_test_attn_stalled takes the arguments of hs_attn_prefill.  In every CTA the warp that issues the
 * first rows' products first waits on an mbarrier that nothing completes; when that wait runs out
 * (1 s, and 20 us for each tile of the call's longest run) the CTA leaves through its abort path, as above,
 * without writing an output of those rows.  Where the call joins partial results, the join runs all the same: with
 * HS_DEVERR_TIMEOUT in d_err the outputs of the rows that it joins mean nothing.
 */
hs_status hs_test_attn_stalled(const hs_attn_shape *shp, const void *q, const void *cache,
                               const int32_t *block_table, void *o, float *lse, const int64_t *pos0,
                               const int32_t *n_tokens, const int64_t *cu_rows, void *workspace,
                               int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream);

/*
 * hs_test_kv8_stalled takes the arguments of hs_kv8_decode.  Every warp that has tiles first waits (1 s) on an mbarrier that
 * nothing completes; it then waits for its own copies, and leaves without a result.  A join runs all the
 * same: with HS_DEVERR_TIMEOUT in d_err none of the outputs means anything.
 */
hs_status hs_test_kv8_stalled(const hs_attn_shape *shp, const void *q, const void *cache,
                              const int32_t *block_table, const int32_t *kv_len, int64_t max_kv_len,
                              void *o, float *lse, void *workspace, int64_t workspace_bytes,
                              int32_t *d_err, cudaStream_t stream);

#ifdef __cplusplus
}
#endif

#endif  // HS_TEST_H
