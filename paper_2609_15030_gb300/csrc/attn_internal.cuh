// Declarations shared by the full-attention calls (attn_api.cu) and their kernels.
#pragma once

#include "hs_attn.h"
#include "hs_internal.cuh"

namespace hs {

// the current device's SM count, queried once per device (hs_api.cu)
hs_status device_sm_count(int *out);

// the release of programmatic dependents alone, for a kernel that has waited before
__device__ __forceinline__ void pdl_release()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// most CTAs of one attention launch
constexpr int kAttnMaxCtas = 320;

// x / d for 0 <= x < 2^31 and 1 <= d < 2^31 as one multiplication: with mul = ceil(2^(31 + s) / d) and
// 2^(s - 1) < d <= 2^s the product is too large by less than x / 2^31 of a 2^s-th, so its floor is x / d.
struct Divisor {
    uint32_t mul, shift;
    int32_t d;
    void set(int32_t by)
    {
        d = by;
        shift = 0;
        while ((int64_t)1 << shift < by)
            ++shift;
        mul = (uint32_t)((((uint64_t)1 << (31 + shift)) + (uint32_t)by - 1) / (uint32_t)by);
    }
    __device__ __forceinline__ int32_t div(int32_t x) const
    {
        return (int32_t)(((uint64_t)(uint32_t)x * mul) >> 31 >> shift);
    }
};

// One attention call, passed by value to the kernels.  A decode step is the call in which every
// request has one token, row b, and the lengths lie on the device.  (What only a prefill needs is a
// parameter of its own: a launch moves all of them.)
struct AttnParams {
    const void *q;
    const void *cache;
    const int32_t *table;         // [batch][max_pages]
    const int32_t *prefix_table;  // decode behind a shared prefix, else nullptr
    const int32_t *kv_len;        // decode: device lengths; prefill: nullptr
    void *o;
    float *lse;                   // or nullptr
    float *part;                  // workspace: partial results (attn_walk.cuh)
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
    int32_t extra;                // units of an item before its tiles: what a segment costs beside them (its
                                  // queries, the ends of its pipeline, its outputs), in tiles
    int32_t extra_shared;         // the same of an item of the shared prefix
    int32_t groups;               // tiles of 128 rows to an item
    int32_t n_split;              // prefill: items that fall to several CTAs
    int32_t parts;                // decode: about the most CTAs that share an item
    int32_t joined;               // partial results are left and joined
    int32_t stall_for_test;       // one wait that nothing completes (failure-detection tests)
    float scale_log2;             // scale * log2(e)
    uint64_t limit_ns;            // after which a wait of the kernel has run out
    Divisor by_group, by_kv;      // group, n_kv
};

// The requests of a prefill, and its schedule.
struct PrefillPlan {
    static constexpr bool kDecode = false;
    struct Request {
        int32_t pos0, n, row0, unused;
    } req[HS_MAX_BATCH];
    struct Cta {                  // where its run of units begins
        int32_t b, item, unit, unused;   // item: row tile * n_kv + KV head; the unit of the item
    } cta[kAttnMaxCtas];
    struct Split {                // an item whose tiles fall to the CTAs c0 to c1
        int32_t item;
        int16_t b, c0, c1, unused;
    } split[kAttnMaxCtas];
};

// a decode step has all of it on the device
struct DecodePlan {
    static constexpr bool kDecode = true;
};

// Host-side checks that the calls share (attn_api.cu): log2 of a page size (-1: not offered); the cache's part of a
// shape; all of it, which fills in the parameters; a decode step's bounds; the pointers; the workspace, which becomes p.part.
int attn_page_shift(int32_t page_size);
hs_status check_attn_cache(const hs_attn_shape &s);
hs_status check_attn_shape(const hs_attn_shape *shp, AttnParams &p);
hs_status check_attn_decode(const hs_attn_shape *shp, int64_t prefix_len, int64_t max_kv_len, AttnParams &p);
hs_status check_attn_pointers(const AttnParams &p, const void *workspace, int64_t workspace_bytes);
hs_status attn_workspace(int64_t need, void *workspace, int64_t workspace_bytes, AttnParams &p);

// Fill in the schedule and say how many bytes of workspace it takes; -1: more units than 31 bits count.
int64_t plan_attn_prefill(AttnParams &p, PrefillPlan &plan, int d, int sm_count);
int64_t plan_attn_decode(AttnParams &p, int d, int sm_count);
cudaError_t launch_attn_prefill(const AttnParams &p, const PrefillPlan &plan, int d, int dtype,
                                cudaStream_t s);
cudaError_t launch_attn_decode(const AttnParams &p, int d, int dtype, cudaStream_t s);
cudaError_t launch_kv_append(const void *k, const void *v, int64_t kv_stride, const int64_t *slots,
                             int64_t n_rows, void *cache, int32_t row_vecs, int32_t page_shift,
                             int64_t num_blocks, int32_t *d_err, int sm_count, cudaStream_t s);

}  // namespace hs
