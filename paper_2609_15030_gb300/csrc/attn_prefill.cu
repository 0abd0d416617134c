// Prefill on the attention kernel (attn_tc.cuh): the schedule, the join of split items and the launches.
#include "attn_tc.cuh"

namespace hs {
namespace attn {
namespace {

// prefill: block (x, y, z) takes 32 rows and 32 columns of the x-th item that is split between CTAs,
// a lane a row and a warp four columns
template <typename T, int D, int NG>
__global__ void __launch_bounds__(kMergeWarps * 32)
attn_merge_prefill_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ PrefillPlan plan)
{
    constexpr int R = 128 * NG, kAhead = 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Start st = find_start<NG>(p, plan, plan.split_at[blockIdx.x]);
    const Walk<NG, PrefillPlan> w(p, plan, nullptr, st);
    const int u0 = st.u - st.at + w.kExtra, u1 = u0 + w.tiles();      // the units of the item's tiles
    const int c0 = cta_of(p.units, p.ctas, u0), c1 = cta_of(p.units, p.ctas, u1 - 1);
    const int64_t size = slot_floats<D>(R);
    const int r = blockIdx.y * 32 + lane, rr = w.rt * R + r, col = blockIdx.z * 32 + warp * 4;
    const bool on = rr < w.rows();
    pdl_wait_and_release();
    if (!on)
        return;
    // part i of the item: CTA c0's last segment, then the first ones of the CTAs behind it
    const float *const first = p.part + (2 * c0 + 1) * size, *const rest = p.part + 2 * c0 * size;
    const int parts = c1 - c0 + 1;
    float m = -INFINITY, l = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < parts; i0 += kAhead) {
        float2 ml[kAhead];
        float v[kAhead][4];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            ml[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[i][e] = 0.f;
            if (i0 + i < parts) {
                const float *const slot = i0 + i == 0 ? first : rest + 2 * (i0 + i) * size;
                ml[i] = reinterpret_cast<const float2 *>(slot)[r];
#pragma unroll
                for (int e = 0; e < 4; ++e)
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
        for (int e = 0; e < 4; ++e)
            a[e] *= f;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            // a part without a key of this row: what it holds of a means nothing
            if (ml[i].x == -INFINITY && ml[i].y == 0.f)
                continue;
            const float h = ex2(ml[i].x - top);
            l = fmaf(ml[i].y, h, l);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                a[e] = fmaf(v[i][e], h, a[e]);
        }
    }
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
    const int t = rr / p.group, head = w.kvh * p.group + rr - t * p.group;
    const int64_t row = plan.req[w.b].row0 + t;
    *reinterpret_cast<uint2 *>(static_cast<T *>(p.o) + row * p.o_stride + head * D + col) =
        make_uint2(Elem<T>::pack(a[0] * inv, a[1] * inv), Elem<T>::pack(a[2] * inv, a[3] * inv));
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
    constexpr int kExtra = extra_units<PrefillPlan, NG>();
    int64_t units = 0;
    for (int b = 0; b < p.batch; ++b)
        for (int rt = 0; rt < row_tiles<NG>(plan.req[b].n * p.group); ++rt)
            units += (int64_t)p.n_kv *
                     (prefill_tiles<NG>(plan.req[b].pos0, plan.req[b].n, p.group, rt) + kExtra);
    if (units > INT_MAX)
        return false;
    p.units = (int)units;
    p.ctas = (int)(units < most ? units : most);
    p.n_split = 0;
    int c = 0;
    int64_t u = 0, split = -1;
    for (int b = 0; b < p.batch && c < p.ctas; ++b)
        for (int rt = 0; rt < row_tiles<NG>(plan.req[b].n * p.group) && c < p.ctas; ++rt) {
            const int n = prefill_tiles<NG>(plan.req[b].pos0, plan.req[b].n, p.group, rt) + kExtra;
            for (; c < p.ctas && first_unit(p.units, p.ctas, c) < u + (int64_t)n * p.n_kv; ++c) {
                const int64_t v = first_unit(p.units, p.ctas, c) - u;
                PrefillPlan::Cta &x = plan.cta[c];
                x.b = b;
                x.item = rt * p.n_kv + (int)(v / n);
                x.unit = (int)(v % n);
                // the first run that begins between an item's tiles names it for the join
                if (x.unit > kExtra && v / n * n + u != split) {
                    split = v / n * n + u;
                    plan.split_at[p.n_split++] = (int16_t)c;
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
    return launch_pdl(attn_merge_prefill_kernel<T, D, NG>, dim3((unsigned)p.n_split, 128 * NG / 32, D / 32),
                      dim3(kMergeWarps * 32), 0, s, p, plan);
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
    return p.joined ? (int64_t)sizeof(float) * 2 * p.ctas * (d == 128 ? slot_floats<128>(rows) : slot_floats<64>(rows))
                    : 0;
}

cudaError_t launch_attn_prefill(const AttnParams &p, const PrefillPlan &plan, int d, int dtype,
                                cudaStream_t s)
{
    return dtype == HS_FP16 ? attn::launch<__half>(p, plan, d, s) : attn::launch<__nv_bfloat16>(p, plan, d, s);
}

}  // namespace hs
