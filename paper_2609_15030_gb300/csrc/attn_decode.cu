// A decode step, with or without a shared prefix, on the attention kernel (attn_tc.cuh): the schedule's
// size, the join of the parts and the launches.
#include "attn_tc.cuh"

namespace hs {
namespace attn {
namespace {

// decode: block (request and KV head, y); with a shared prefix its parts first
template <typename T, int D, int NG>
__global__ void __launch_bounds__(kMergeWarps * 32)
attn_merge_decode_kernel(const __grid_constant__ AttnParams p, int per_row)
{
    __shared__ int32_t len[HS_MAX_BATCH];
    __shared__ int sums[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = blockIdx.x / p.n_kv, kvh = blockIdx.x - b * p.n_kv;
    // the lengths may be read before the wait: the kernel in front, which has waited itself, only
    // reads them
    if (warp == 0) {
        int before = 0;
        const int n = read_lengths(p, len, lane, false, b, &before);
        if (lane == 0) {
            sums[0] = before;
            sums[1] = n;
        }
    }
    __syncthreads();
    const int per = prefix_units(p), own = item_units(p, len[b]);
    const int pre = per * p.n_kv * row_tiles<NG>(p.batch * p.group);
    const int units = pre + sums[1];
    const int u0 = pre + sums[0] + kvh * own;
    const int item = b * p.n_kv + kvh;
    const bool skip = len[b] < 0;
    // an unsplit item belongs to the CTA in whose run it begins, else the CTAs with its tiles have it
    const int c0 = skip ? 0 : cta_of(units, p.ctas, p.unsplit ? u0 : u0 + p.extra);
    const int c1 = skip || p.unsplit ? c0 : cta_of(units, p.ctas, u0 + own - 1);
    pdl_wait_and_release();
    if (skip || (per == 0 && c0 == c1))
        return;
    const int64_t own_at = per > 0 ? prefix_part_floats<D, NG>(p) : 0, size = slot_floats<D>(p.group);
    const int64_t pre_size = slot_floats<D>(128 * NG);
    const int some = kMergeWarps / per_row;
    for (int h0 = blockIdx.y * some; h0 < p.group; h0 += gridDim.y * some) {
        const int h = h0 + warp / per_row;
        const bool on = h < p.group;
        const int rr = b * p.group + h, rt = rr / (128 * NG), r = rr - rt * 128 * NG;
        const int pitem = rt * p.n_kv + kvh;
        int p0 = 0, p1 = -1;
        if (on && per > 0) {
            p0 = cta_of(units, p.ctas, pitem * per + (p.unsplit ? 0 : p.extra_shared));
            p1 = p.unsplit ? p0 : cta_of(units, p.ctas, (pitem + 1) * per - 1);
        }
        const int n = p1 - p0 + 1;
        const Joined<D> x = join_parts<D>(
            p.part, on ? n + c1 - c0 + 1 : 0, warp % per_row, per_row, lane,
            [&](int i, int64_t &at_pair, int64_t &at_a) {
                const bool pre_part = i < n;
                const int c = pre_part ? p0 + i : c0 + i - n;
                const int64_t slot =
                    pre_part ? (pitem + c) * pre_size
                    : per > 0 ? own_at + (item + c) * size
                              : (int64_t)(c == c0 ? 2 * c + 1 : 2 * c) * size;
                const int row = pre_part ? r : h;
                at_pair = slot + 2 * row;
                at_a = slot + pairs_floats(pre_part ? 128 * NG : p.group) + (int64_t)row * D;
                return has_units(units, p.ctas, c);
            });
        finish_row<T, D>(p, x, per_row, warp, lane, on, b, kvh * p.group + h);
    }
}

template <typename T, int D, int NG>
cudaError_t launch(const AttnParams &p, cudaStream_t s)
{
    const cudaError_t e = launch_tc<T, D, NG>(p, DecodePlan{}, s);
    if (e != cudaSuccess || !p.joined)
        return e;
    // warps to a row: about eight parts each
    int per_row = 1;
    while (per_row < kMergeWarps && per_row * 8 < p.parts)
        per_row *= 2;
    const unsigned y = (unsigned)((p.group * per_row + kMergeWarps - 1) / kMergeWarps);
    return launch_pdl(attn_merge_decode_kernel<T, D, NG>, dim3((unsigned)(p.batch * p.n_kv), y),
                      dim3(kMergeWarps * 32), 0, s, p, per_row);
}

template <typename T>
cudaError_t launch(const AttnParams &p, int d, cudaStream_t s)
{
    if (p.groups == 2)
        return d == 128 ? launch<T, 128, 2>(p, s) : launch<T, 64, 2>(p, s);
    return d == 128 ? launch<T, 128, 1>(p, s) : launch<T, 64, 1>(p, s);
}

}  // namespace
}  // namespace attn

int64_t plan_attn_decode(AttnParams &p, int d, int sm_count)
{
    using namespace attn;
    // two tiles of rows to an item where the rows in front of a shared prefix fill them
    p.groups = p.prefix_len > 0 && p.batch * p.group > 128 ? 2 : 1;
    int most = sm_count * (p.groups == 2 ? 1 : 2);
    if (most > kAttnMaxCtas)
        most = kAttnMaxCtas;
    auto slot = [&](int rows) {
        return (int64_t)sizeof(float) * (d == 128 ? slot_floats<128>(rows) : slot_floats<64>(rows));
    };
    const int own_tiles = p.max_kv > 0 ? tiles_of(p.max_kv) : 1, shared_tiles = tiles_of(p.prefix_len);
    const int rows = p.batch * p.group;
    const int64_t own = (int64_t)p.batch * p.n_kv;
    const int64_t shared = p.prefix_len == 0 ? 0 : (int64_t)p.n_kv *
                           (p.groups == 2 ? row_tiles<2>(rows) : row_tiles<1>(rows));
    // What a segment costs beside its tiles.  32 ragged requests: 53.6 us with 1 where 0 took 55; behind a
    // shared prefix, 32 requests of a tile each 22.9 us with 1 instead of 26.5, but where two tiles of rows
    // take a CTA's own items in turn, 384 requests 96 us with 0 instead of 120.  A prefix's items end
    // with the sums of all requests' rows: 64 requests behind 32,768 keys 64.2 us with 4 where 0 took 68.3,
    // but 8 behind 4,608, less than a tile to a CTA, 11.2 us with 0 instead of 11.8 with 4.
    const int64_t share = (own * own_tiles + shared * shared_tiles) / most;
    p.extra = p.prefix_len == 0 || (p.groups == 1 && share >= 2) ? 1 : 0;
    p.extra_shared = (int)(share / 2 < 4 ? share / 2 : 4);
    const int64_t units = own * (own_tiles + p.extra) + shared * prefix_units(p);
    if (units > INT_MAX)
        return -1;
    p.ctas = (int)(units < most ? units : most);
    const int longest = tiles_of(p.max_kv > p.prefix_len ? p.max_kv : p.prefix_len);
    p.limit_ns = wait_limit_ns(p, longest, units);
    p.parts = (int)(longest / (units / p.ctas > 0 ? units / p.ctas : 1)) + 2;
    if (p.prefix_len > 0) {
        p.joined = 1;
        return (shared + p.ctas) * slot(128 * p.groups) + (own + p.ctas) * slot(p.group);
    }
    // The lengths are known on the device alone, and max_kv is only their bound: one request may have that many
    // keys and the others none.  So an even share is counted as if every item had a tile, which leaves whole
    // items to bounds of 3 tiles (4 with an item or less to a CTA).  38 requests of 8 KV heads, an item to a CTA:
    // with one at 131,072 keys and the others at 100, 96 us where whole items took 1,380; with all at 4,096, 96.4
    // instead of 95.5, of 37 requests 97 to 100 instead of 92 to 93; at 300 keys under a bound of 131,072, 12.8
    // instead of 11.7 (the join's launch).
    if (better_whole(p, own, own_tiles, own * (1 + p.extra)))
        p.unsplit = 1;
    p.joined = !p.unsplit;
    return p.joined ? 2 * p.ctas * slot(p.group) : 0;
}

cudaError_t launch_attn_decode(const AttnParams &p, int d, int dtype, cudaStream_t s)
{
    return dtype == HS_FP16 ? attn::launch<__half>(p, d, s) : attn::launch<__nv_bfloat16>(p, d, s);
}

}  // namespace hs
