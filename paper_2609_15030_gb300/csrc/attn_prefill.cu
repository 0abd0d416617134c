// Prefill on the attention kernel (attn_tc.cuh): the schedule, the join of split items and the launches.
#include "attn_tc.cuh"

namespace hs {
namespace attn {
namespace {

// Block (x, y, z) takes 32 rows and 8 E columns of the x-th item that is split between CTAs, a lane a row
// and a warp E columns: 4 where few items are split (of many parts each), all of them in one block where more
// than 64 are.  Tails of 200 to 260 tokens behind 3,000 and more keys, 16 heads over 4 of 128, the whole call: 16
// split items 15.3 us (16.9 in one block each), 64 32.2 (30.2), 80 38.1 (35.9), 137 65.7 (60.9); heads of 64 with
// 64 items 23.8 (23.1), of 128 with one tile of rows to an item 31.0 (32.0).
template <typename T, int D, int NG, int E>
__global__ void __launch_bounds__(kMergeWarps * 32)
attn_merge_prefill_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ PrefillPlan plan)
{
    constexpr int R = 128 * NG, kAhead = 32 / E;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const PrefillPlan::Split it = plan.split[blockIdx.x];
    const int rt = p.by_kv.div(it.item), kvh = it.item - rt * p.n_kv;
    const int64_t size = slot_floats<D>(R);
    const int r = blockIdx.y * 32 + lane, rr = rt * R + r, col = (blockIdx.z * kMergeWarps + warp) * E;
    const bool on = rr < plan.req[it.b].n * p.group;
    const int t = p.by_group.div(on ? rr : 0), head = kvh * p.group + rr - t * p.group;
    const int64_t row = plan.req[it.b].row0 + t;
    pdl_wait_and_release();
    if (!on)
        return;
    // part i of the item: CTA c0's last segment, then the first ones of the CTAs behind it
    const float *const first = p.part + (2 * it.c0 + 1) * size, *const rest = p.part + 2 * it.c0 * size;
    const int parts = it.c1 - it.c0 + 1;
    float m = -INFINITY, l = 0.f, a[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
        a[e] = 0.f;
    for (int i0 = 0; i0 < parts; i0 += kAhead) {
        float2 ml[kAhead];
        float v[kAhead][E];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            ml[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[i][e] = 0.f;
            if (i0 + i < parts) {
                const float *const slot = i0 + i == 0 ? first : rest + 2 * (i0 + i) * size;
                ml[i] = reinterpret_cast<const float2 *>(slot)[r];
#pragma unroll
                for (int e = 0; e < E; ++e)
                    v[i][e] = slot[pairs_floats(R) + (col + e) * R + r];
            }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            top = fmaxf(top, ml[i].x);
        const float f = m == -INFINITY && l == 0.f ? 0.f : ex2(m - top);
        m = top;
        l *= f;
#pragma unroll
        for (int e = 0; e < E; ++e)
            a[e] *= f;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            // a part without a key of this row: what it holds of a means nothing
            if (ml[i].x == -INFINITY && ml[i].y == 0.f)
                continue;
            const float h = ex2(ml[i].x - top);
            l = fmaf(ml[i].y, h, l);
#pragma unroll
            for (int e = 0; e < E; ++e)
                a[e] = fmaf(v[i][e], h, a[e]);
        }
    }
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
    T *const o = static_cast<T *>(p.o) + row * p.o_stride + head * D + col;
#pragma unroll
    for (int e = 0; e < E; ++e)
        a[e] = Elem<T>::in_range(a[e] * inv);
#pragma unroll
    for (int e = 0; e < E; e += 4)
        *reinterpret_cast<uint2 *>(o + e) = make_uint2(Elem<T>::pack(a[e], a[e + 1]),
                                                       Elem<T>::pack(a[e + 2], a[e + 3]));
    if (p.lse != nullptr && col == 0)
        p.lse[row * p.n_heads + head] = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
}

// ---- the schedule --------------------------------------------------------------------------

// tiles of rows of an item: two where a request has them
int groups_of(const AttnParams &p, const PrefillPlan &plan)
{
    int most = 0;
    for (int b = 0; b < p.batch; ++b)
        most = plan.req[b].n > most ? plan.req[b].n : most;
    return most * p.group > 128 ? 2 : 1;
}

template <int NG>
bool schedule(AttnParams &p, PrefillPlan &plan, int most)
{
    // With 1 CTAs with many short items end long after the others (nine packed tails 53.9 us, two 8k-token
    // prompts of 64-wide heads 590); 2 take 50.5 and 515, 3 take 51.7 and 515, 4 53.0 and 521.
    p.extra = 2;
    int64_t units = 0, items = 0;
    int longest = 0;
    for (int b = 0; b < p.batch; ++b)
        for (int rt = 0; rt < row_tiles<NG>(plan.req[b].n * p.group); ++rt) {
            const int n = prefill_tiles<NG>(plan.req[b].pos0, plan.req[b].n, p.group, rt) + p.extra;
            units += (int64_t)p.n_kv * n;
            items += p.n_kv;
            longest = n > longest ? n : longest;
            if (units > INT_MAX)
                return false;
        }
    p.units = (int)units;
    p.ctas = (int)(units < most ? units : most);
    p.limit_ns = wait_limit_ns(p, longest, units);
    p.n_split = 0;
    if (better_whole(p, items, longest - p.extra, units))
        p.unsplit = 1;
    int c = 0;
    int64_t u = 0, split = -1;
    for (int b = 0; b < p.batch && c < p.ctas; ++b)
        for (int rt = 0; rt < row_tiles<NG>(plan.req[b].n * p.group) && c < p.ctas; ++rt) {
            const int n = prefill_tiles<NG>(plan.req[b].pos0, plan.req[b].n, p.group, rt) + p.extra;
            for (; c < p.ctas && first_unit(p.units, p.ctas, c) < u + (int64_t)n * p.n_kv; ++c) {
                const int64_t v = first_unit(p.units, p.ctas, c) - u;
                PrefillPlan::Cta &x = plan.cta[c];
                x.b = b;
                x.item = rt * p.n_kv + (int)(v / n);
                x.unit = (int)(v % n);
                // a run that begins between an item's tiles: the item is split
                const int64_t item = u + v / n * n;
                if (x.unit > p.extra && item != split) {
                    split = item;
                    PrefillPlan::Split &y = plan.split[p.n_split++];
                    y.item = x.item;
                    y.b = (int16_t)b;
                    y.c0 = (int16_t)cta_of(p.units, p.ctas, (int)item + p.extra);
                    y.c1 = (int16_t)cta_of(p.units, p.ctas, (int)item + n - 1);
                }
            }
            u += (int64_t)n * p.n_kv;
        }
    return true;
}

template <typename T, int D, int NG>
cudaError_t launch(const AttnParams &p, const PrefillPlan &plan, cudaStream_t s)
{
    const cudaError_t e = launch_tc<T, D, NG>(p, plan, s);
    if (e != cudaSuccess || !p.joined)
        return e;
    if (p.n_split > 64)
        return launch_pdl(attn_merge_prefill_kernel<T, D, NG, D / kMergeWarps>,
                          dim3((unsigned)p.n_split, 128 * NG / 32), dim3(kMergeWarps * 32), 0, s, p, plan);
    return launch_pdl(attn_merge_prefill_kernel<T, D, NG, 4>,
                      dim3((unsigned)p.n_split, 128 * NG / 32, D / 32), dim3(kMergeWarps * 32), 0, s, p, plan);
}

template <typename T>
cudaError_t launch(const AttnParams &p, const PrefillPlan &plan, int d, cudaStream_t s)
{
    if (p.groups == 2)
        return d == 128 ? launch<T, 128, 2>(p, plan, s) : launch<T, 64, 2>(p, plan, s);
    return d == 128 ? launch<T, 128, 1>(p, plan, s) : launch<T, 64, 1>(p, plan, s);
}

}  // namespace
}  // namespace attn

int64_t plan_attn_prefill(AttnParams &p, PrefillPlan &plan, int d, int sm_count)
{
    using namespace attn;
    p.groups = groups_of(p, plan);
    int most = sm_count * (p.groups == 2 ? 1 : 2);
    if (most > kAttnMaxCtas)
        most = kAttnMaxCtas;
    if (!(p.groups == 2 ? schedule<2>(p, plan, most) : schedule<1>(p, plan, most)))
        return -1;
    p.joined = !p.unsplit && p.n_split > 0;
    const int rows = 128 * p.groups;
    const int64_t slot = (int64_t)sizeof(float) * (d == 128 ? slot_floats<128>(rows) : slot_floats<64>(rows));
    return p.joined ? 2 * p.ctas * slot : 0;
}

cudaError_t launch_attn_prefill(const AttnParams &p, const PrefillPlan &plan, int d, int dtype,
                                cudaStream_t s)
{
    return dtype == HS_FP16 ? attn::launch<__half>(p, plan, d, s) : attn::launch<__nv_bfloat16>(p, plan, d, s);
}

}  // namespace hs
