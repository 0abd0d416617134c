// C-ABI entry points of the full-attention calls: host-side validation, then the launches.
// Validation happens before any CUDA runtime call, so argument errors are reported without
// touching the GPU.
#include <cmath>
#include <cstring>

#include "attn_internal.cuh"
#include "hs_test.h"

namespace {

inline bool misaligned16(const void *p)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) != 0;
}

inline hs_status cuda_status(cudaError_t e)
{
    return e == cudaSuccess ? HS_OK : HS_ERR_CUDA;
}

int page_shift(int32_t page_size)
{
    for (int s = 4; s <= 8; ++s)
        if (page_size == 1 << s)
            return s;
    return -1;
}

// what every call asks of the cache's part of the shape
hs_status check_cache(const hs_attn_shape &s)
{
    if (s.n_kv_heads < 1 || s.num_blocks < 0 || s.page_size < 1)
        return HS_ERR_INVALID_ARG;
    if (s.dtype != HS_BF16 && s.dtype != HS_FP16)
        return HS_ERR_INVALID_ARG;
    if ((s.head_dim != 64 && s.head_dim != 128) || page_shift(s.page_size) < 0)
        return HS_ERR_UNSUPPORTED;
    // the cache's rows of 64 elements are counted in 32 bits
    if (s.n_kv_heads > 1024 || s.num_blocks > INT32_MAX / (2 * (s.page_size / 8)))
        return HS_ERR_UNSUPPORTED;
    return HS_OK;
}

hs_status check_shape(const hs_attn_shape *shp, hs::AttnParams &p)
{
    if (shp == nullptr)
        return HS_ERR_INVALID_ARG;
    const hs_attn_shape s = *shp;
    const hs_status st = check_cache(s);
    if (st == HS_ERR_INVALID_ARG)
        return st;
    if (s.batch < 0 || s.n_heads < 1 || s.n_heads % s.n_kv_heads != 0 || s.max_pages < 0 ||
        s.q_stride < 0 || s.o_stride < 0 || !(s.scale > 0.f) || !std::isfinite(s.scale) ||
        (s.unsplit != 0 && s.unsplit != 1))
        return HS_ERR_INVALID_ARG;
    if (st != HS_OK)
        return st;
    if (s.batch > HS_MAX_BATCH || s.n_heads / s.n_kv_heads > 128 || s.q_stride > INT32_MAX ||
        s.o_stride > INT32_MAX)
        return HS_ERR_UNSUPPORTED;
    const int64_t inner = (int64_t)s.n_heads * s.head_dim;
    if ((s.q_stride != 0 && s.q_stride < inner) || (s.o_stride != 0 && s.o_stride < inner))
        return HS_ERR_INVALID_ARG;
    if (s.q_stride % 8 != 0 || s.o_stride % 8 != 0)
        return HS_ERR_MISALIGNED;
    std::memset(&p, 0, sizeof p);
    p.num_blocks = s.num_blocks;
    p.max_pages = s.max_pages;
    p.q_stride = s.q_stride != 0 ? s.q_stride : inner;
    p.o_stride = s.o_stride != 0 ? s.o_stride : inner;
    p.batch = s.batch;
    p.n_heads = s.n_heads;
    p.n_kv = s.n_kv_heads;
    p.group = s.n_heads / s.n_kv_heads;
    p.by_group.set(p.group);
    p.by_kv.set(p.n_kv);
    p.page_shift = page_shift(s.page_size);
    p.unsplit = s.unsplit;
    p.scale_log2 = s.scale * 1.4426950408889634f;
    return HS_OK;
}

hs_status room(int64_t need, void *workspace, int64_t workspace_bytes, hs::AttnParams &p)
{
    if (need < 0)
        return HS_ERR_UNSUPPORTED;
    if (need > workspace_bytes || (need > 0 && workspace == nullptr))
        return HS_ERR_INVALID_ARG;
    p.part = static_cast<float *>(workspace);
    return HS_OK;
}

// the requests' lengths into the plan; *any: whether there is a token
hs_status check_lengths(const hs_attn_shape &s, const int64_t *pos0, const int32_t *n_tokens,
                        const int64_t *cu_rows, bool rows, const hs::AttnParams &p,
                        hs::PrefillPlan &plan, bool *any)
{
    *any = false;
    if (s.batch == 0)
        return HS_OK;
    if (pos0 == nullptr || n_tokens == nullptr || (rows && cu_rows == nullptr))
        return HS_ERR_INVALID_ARG;
    const int64_t room = s.max_pages > INT32_MAX ? INT64_MAX : s.max_pages * s.page_size;
    for (int32_t b = 0; b < s.batch; ++b) {
        if (pos0[b] < 0 || n_tokens[b] < 0 || pos0[b] > ((int64_t)1 << 40))
            return HS_ERR_INVALID_ARG;
        if (n_tokens[b] > 0 && pos0[b] + n_tokens[b] > room)
            return HS_ERR_INVALID_ARG;
        if (rows && (cu_rows[b] < 0 || cu_rows[b + 1] < cu_rows[b] ||
                     n_tokens[b] > cu_rows[b + 1] - cu_rows[b]))
            return HS_ERR_INVALID_ARG;
    }
    for (int32_t b = 0; b < s.batch; ++b) {
        plan.req[b] = {};
        if (n_tokens[b] == 0)
            continue;
        *any = true;
        if (pos0[b] + n_tokens[b] > INT32_MAX - 8192 ||
            (int64_t)n_tokens[b] * p.group > INT32_MAX - 8192 ||
            (rows && cu_rows[b] + n_tokens[b] > INT32_MAX / p.n_heads))
            return HS_ERR_UNSUPPORTED;
        plan.req[b].pos0 = (int32_t)pos0[b];
        plan.req[b].n = n_tokens[b];
        plan.req[b].row0 = rows ? (int32_t)cu_rows[b] : 0;
    }
    return HS_OK;
}

hs_status check_pointers(const hs::AttnParams &p, const void *workspace, int64_t workspace_bytes)
{
    if (p.q == nullptr || p.cache == nullptr || p.table == nullptr || p.o == nullptr ||
        workspace_bytes < 0 || p.num_blocks < 1)
        return HS_ERR_INVALID_ARG;
    if (misaligned16(p.q) || misaligned16(p.cache) || misaligned16(p.o) || misaligned16(workspace) ||
        (reinterpret_cast<uintptr_t>(p.table) & 3u) != 0 ||
        (reinterpret_cast<uintptr_t>(p.lse) & 3u) != 0)
        return HS_ERR_MISALIGNED;
    return HS_OK;
}

hs_status check_decode(const hs_attn_shape *shp, int64_t prefix_len, int64_t max_kv_len,
                       hs::AttnParams &p)
{
    const hs_status st = check_shape(shp, p);
    if (st != HS_OK)
        return st;
    const int64_t room = shp->max_pages > INT32_MAX ? INT64_MAX : shp->max_pages * shp->page_size;
    if (prefix_len < 0 || max_kv_len < 0 || max_kv_len > room)
        return HS_ERR_INVALID_ARG;
    if (prefix_len > INT32_MAX - 8192 || max_kv_len > INT32_MAX - 8192 - prefix_len)
        return HS_ERR_UNSUPPORTED;
    p.max_kv = (int32_t)max_kv_len;
    p.prefix_len = (int32_t)prefix_len;
    return HS_OK;
}

hs_status decode(const hs_attn_shape *shp, const void *q, const void *cache,
                 const int32_t *prefix_table, int64_t prefix_len, const int32_t *block_table,
                 const int32_t *kv_len, int64_t max_kv_len, void *o, float *lse, void *workspace,
                 int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream)
{
    hs::AttnParams p;
    hs_status st = check_decode(shp, prefix_len, max_kv_len, p);
    if (st != HS_OK)
        return st;
    if (p.batch == 0)
        return HS_OK;
    if (kv_len == nullptr || (prefix_len > 0 && prefix_table == nullptr))
        return HS_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(kv_len) | reinterpret_cast<uintptr_t>(prefix_table)) & 3u) != 0)
        return HS_ERR_MISALIGNED;
    p.q = q;
    p.cache = cache;
    p.table = block_table;
    p.prefix_table = prefix_table;
    p.kv_len = kv_len;
    p.o = o;
    p.lse = lse;
    p.d_err = d_err;
    st = check_pointers(p, workspace, workspace_bytes);
    if (st != HS_OK)
        return st;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st == HS_OK)
        st = room(hs::plan_attn_decode(p, shp->head_dim, sms), workspace, workspace_bytes, p);
    if (st != HS_OK)
        return st;
    return cuda_status(hs::launch_attn_decode(p, shp->head_dim, shp->dtype, stream));
}

}  // namespace

extern "C" {

hs_status hs_kv_append(const hs_attn_shape *shp, const void *k, const void *v, int64_t kv_stride,
                       const int64_t *slots, int64_t n_rows, void *cache, int32_t *d_err,
                       cudaStream_t stream)
{
    if (shp == nullptr || n_rows < 0 || kv_stride < 0)
        return HS_ERR_INVALID_ARG;
    hs_status st = check_cache(*shp);
    if (st != HS_OK)
        return st;
    const int64_t inner = (int64_t)shp->n_kv_heads * shp->head_dim;
    if (kv_stride != 0 && kv_stride < inner)
        return HS_ERR_INVALID_ARG;
    if (kv_stride % 8 != 0)
        return HS_ERR_MISALIGNED;
    if (n_rows == 0)
        return HS_OK;
    if (k == nullptr || v == nullptr || slots == nullptr || cache == nullptr)
        return HS_ERR_INVALID_ARG;
    if (misaligned16(k) || misaligned16(v) || misaligned16(cache) ||
        (reinterpret_cast<uintptr_t>(slots) & 7u) != 0)
        return HS_ERR_MISALIGNED;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st != HS_OK)
        return st;
    return cuda_status(hs::launch_kv_append(k, v, kv_stride != 0 ? kv_stride : inner, slots, n_rows,
                                            cache, (int32_t)(inner / 8), page_shift(shp->page_size),
                                            shp->num_blocks, d_err, sms, stream));
}

static hs_status prefill(const hs_attn_shape *shp, const void *q, const void *cache,
                         const int32_t *block_table, void *o, float *lse, const int64_t *pos0,
                         const int32_t *n_tokens, const int64_t *cu_rows, void *workspace,
                         int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream,
                         bool stall_for_test)
{
    hs::AttnParams p;
    hs::PrefillPlan plan;
    hs_status st = check_shape(shp, p);
    bool any = false;
    if (st == HS_OK)
        st = check_lengths(*shp, pos0, n_tokens, cu_rows, true, p, plan, &any);
    if (st != HS_OK || !any)
        return st;
    p.q = q;
    p.cache = cache;
    p.table = block_table;
    p.o = o;
    p.lse = lse;
    p.d_err = d_err;
    p.stall_for_test = stall_for_test;
    st = check_pointers(p, workspace, workspace_bytes);
    if (st != HS_OK)
        return st;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st == HS_OK)
        st = room(hs::plan_attn_prefill(p, plan, shp->head_dim, sms), workspace, workspace_bytes, p);
    if (st != HS_OK)
        return st;
    return cuda_status(hs::launch_attn_prefill(p, plan, shp->head_dim, shp->dtype, stream));
}

hs_status hs_attn_prefill(const hs_attn_shape *shp, const void *q, const void *cache,
                          const int32_t *block_table, void *o, float *lse, const int64_t *pos0,
                          const int32_t *n_tokens, const int64_t *cu_rows, void *workspace,
                          int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream)
{
    return prefill(shp, q, cache, block_table, o, lse, pos0, n_tokens, cu_rows, workspace, workspace_bytes,
                   d_err, stream, false);
}

hs_status hs_test_attn_stalled(const hs_attn_shape *shp, const void *q, const void *cache,
                               const int32_t *block_table, void *o, float *lse, const int64_t *pos0,
                               const int32_t *n_tokens, const int64_t *cu_rows, void *workspace,
                               int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream)
{
    return prefill(shp, q, cache, block_table, o, lse, pos0, n_tokens, cu_rows, workspace, workspace_bytes,
                   d_err, stream, true);
}

hs_status hs_attn_prefill_workspace_bytes(const hs_attn_shape *shp, const int64_t *pos0,
                                          const int32_t *n_tokens, int64_t *bytes_out)
{
    if (bytes_out == nullptr)
        return HS_ERR_INVALID_ARG;
    hs::AttnParams p;
    hs::PrefillPlan plan;
    hs_status st = check_shape(shp, p);
    bool any = false;
    if (st == HS_OK)
        st = check_lengths(*shp, pos0, n_tokens, nullptr, false, p, plan, &any);
    if (st != HS_OK)
        return st;
    *bytes_out = 0;
    if (!any)
        return HS_OK;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st != HS_OK)
        return st;
    const int64_t need = hs::plan_attn_prefill(p, plan, shp->head_dim, sms);
    if (need < 0)
        return HS_ERR_UNSUPPORTED;
    *bytes_out = need;
    return HS_OK;
}

hs_status hs_attn_decode(const hs_attn_shape *shp, const void *q, const void *cache,
                         const int32_t *block_table, const int32_t *kv_len, int64_t max_kv_len,
                         void *o, float *lse, void *workspace, int64_t workspace_bytes,
                         int32_t *d_err, cudaStream_t stream)
{
    return decode(shp, q, cache, nullptr, 0, block_table, kv_len, max_kv_len, o, lse, workspace,
                  workspace_bytes, d_err, stream);
}

hs_status hs_attn_decode_shared(const hs_attn_shape *shp, const void *q, const void *cache,
                                const int32_t *prefix_table, int64_t prefix_len,
                                const int32_t *block_table, const int32_t *kv_len,
                                int64_t max_kv_len, void *o, float *lse, void *workspace,
                                int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream)
{
    return decode(shp, q, cache, prefix_table, prefix_len, block_table, kv_len, max_kv_len, o, lse,
                  workspace, workspace_bytes, d_err, stream);
}

hs_status hs_attn_decode_workspace_bytes(const hs_attn_shape *shp, int64_t max_kv_len,
                                         int64_t *bytes_out)
{
    return hs_attn_decode_shared_workspace_bytes(shp, 0, max_kv_len, bytes_out);
}

hs_status hs_attn_decode_shared_workspace_bytes(const hs_attn_shape *shp, int64_t prefix_len,
                                                int64_t max_kv_len, int64_t *bytes_out)
{
    if (bytes_out == nullptr)
        return HS_ERR_INVALID_ARG;
    hs::AttnParams p;
    hs_status st = check_decode(shp, prefix_len, max_kv_len, p);
    if (st != HS_OK)
        return st;
    *bytes_out = 0;
    if (p.batch == 0)
        return HS_OK;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st != HS_OK)
        return st;
    const int64_t need = hs::plan_attn_decode(p, shp->head_dim, sms);
    if (need < 0)
        return HS_ERR_UNSUPPORTED;
    *bytes_out = need;
    return HS_OK;
}

}  // extern "C"
