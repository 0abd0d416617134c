// Declarations shared by the full-attention calls (attn_api.cu) and their kernels.
#pragma once

#include "hs_internal.cuh"

namespace hs {

// most CTAs of one attention launch
constexpr int kAttnMaxCtas = 320;

// One attention call, passed by value to the kernels.  A decode step is the call in which every
// request has one token, row b, and the lengths lie on the device.
struct AttnParams {
    const void *q;
    const void *cache;
    const int32_t *table;         // [batch][max_pages]
    const int32_t *prefix_table;  // decode behind a shared prefix, else nullptr
    const int32_t *kv_len;        // decode: device lengths; prefill: nullptr
    void *o;
    float *lse;                   // or nullptr
    float *part;                  // workspace: partial results (see attn.cu)
    int32_t *d_err;
    int64_t num_blocks;
    int64_t max_pages;
    int64_t q_stride;
    int64_t o_stride;
    int32_t batch;
    int32_t n_heads;
    int32_t n_kv;
    int32_t group;                // n_heads / n_kv
    int32_t page_shift;           // log2(page_size)
    int32_t max_kv;               // decode: bound of kv_len
    int32_t prefix_len;
    int32_t unsplit;
    int32_t units;                // prefill: key tiles of all items
    int32_t ctas;
    int32_t parts;                // about the most CTAs that share an item
    int32_t joined;               // partial results are left and joined
    float scale_log2;             // scale * log2(e)
    // prefill only: the requests, and where each CTA's share of the tiles begins
    int32_t pos0[HS_MAX_BATCH];
    int32_t n_tokens[HS_MAX_BATCH];
    int32_t row0[HS_MAX_BATCH];
    int32_t start_item[kAttnMaxCtas];   // row tile * n_kv + KV head of the request
    int32_t start_kt[kAttnMaxCtas];
    int16_t start_b[kAttnMaxCtas];
    int16_t split_at[kAttnMaxCtas];     // CTAs whose run is the first to begin inside an item
    int32_t n_split;
};

// Fills in the schedule (units, ctas, start_*) and says how many bytes of workspace it takes; -1: more
// units than 31 bits count.
int64_t plan_attn(AttnParams &p, int d, int sm_count);
cudaError_t launch_attn(const AttnParams &p, int d, int dtype, cudaStream_t s);
cudaError_t launch_kv_append(const void *k, const void *v, int64_t kv_stride, const int64_t *slots,
                             int64_t n_rows, void *cache, int32_t row_vecs, int32_t page_shift,
                             int64_t num_blocks, int32_t *d_err, int sm_count, cudaStream_t s);

}  // namespace hs
