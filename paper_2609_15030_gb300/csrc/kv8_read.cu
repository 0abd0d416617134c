// A prefix of the 8-bit cache read back into 16-bit pages, where a prefill finds it (the restored entries that the
// recomputed suffix attends to, Section 2.2 of the paper).
//
// Bytes in, twice as many out: bound by HBM.  Units of 16 tokens (a group, all heads, both planes) are shared
// out evenly over the blocks, whatever the requests' lengths.  A thread takes 16 bytes of a token to 32, of up to
// eight (KV head, plane) at a time.  459,413 tokens of 8 heads of 128 (2.82 GB) take 435 us, 6.5 TB/s; with 8 bytes to
// 16 and as many loads in flight 6 % more.  Groups of fewer heads have fewer loads for a thread (16 requests of 3,000 tokens of 4
// heads: 26 us, 5.5 TB/s); taking several groups at a time, each vector with its own table entries, cost more than it
// brought (35 us).
#include "kv8_walk.cuh"

namespace hs {
namespace {

using namespace kv8;

constexpr int kThreads = 256;

// 32 bytes, in one store where the address is a multiple of that
__device__ __forceinline__ void store(uint4 *to, bool wide, uint4 a, uint4 b)
{
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(a.x), "r"(a.y), "r"(a.z),
                     "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                     : "memory");
    } else {
        to[0] = a;
        to[1] = b;
    }
}

template <typename T, int D, int kAhead>
__global__ void __launch_bounds__(kThreads)
kv8_read_kernel(const __grid_constant__ Kv8Read p)
{
    constexpr int kVecs = D / 16;                         // 16-byte vectors of a token
    constexpr int kPieces = kThreads / (kGroup * kVecs);  // (KV head, plane) pairs of a block at a time
    __shared__ Lengths all;
    pdl_wait_and_release();
    const int lane = threadIdx.x & 31;
    read_lengths(all, p.kv_len, p.batch, p.max_kv, p.d_err, [](int len) { return groups_of(len); });
    const int64_t units = all.before[p.batch];
    int u = (int)(units * blockIdx.x / gridDim.x);
    const int end = (int)(units * (blockIdx.x + 1) / gridDim.x);
    if (u >= end)
        return;
    int b = request_of(all, p.batch, u, lane);
    const int piece = threadIdx.x / (kGroup * kVecs), token = threadIdx.x / kVecs % kGroup,
              vec = threadIdx.x % kVecs;
    const int shift = p.cache.page_shift - 4;
    const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31) == 0;     // rows of a head are multiples of 32 bytes
    for (; u < end; ++u) {
        while (all.before[b + 1] <= u)
            ++b;
        const int g = u - all.before[b];
        const int64_t entry = (int64_t)b * p.max_pages + (g >> shift);
        const int from = __ldg(p.table + entry), to = __ldg(p.out_table + entry);
        if (from < 0 || from >= p.cache.num_blocks || to < 0 || to >= p.out_blocks) {
            if (threadIdx.x == 0)
                report(p.d_err, HS_DEVERR_BLOCK_OOB);
            continue;
        }
        const bool on = g * kGroup + token < all.len[b];
        const int in_page = g & ((1 << shift) - 1);
        uint4 *const out = p.out + (((int64_t)to * 2 << p.cache.page_shift) + in_page * kGroup + token) *
                                       p.cache.n_kv * (2 * kVecs) + 2 * vec;
        for (int i0 = piece; i0 < 2 * p.cache.n_kv; i0 += kPieces * kAhead) {
            uint4 x[kAhead];
            float scale[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int head_plane = i0 + i * kPieces;
                if (head_plane >= 2 * p.cache.n_kv || !on)
                    continue;
                float *at_scale;
                const uint8_t *const at = group_at<D>(p.cache, from, in_page, head_plane, &at_scale);
                x[i] = __ldcs(reinterpret_cast<const uint4 *>(at + token * D) + vec);
                scale[i] = __ldg(at_scale);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int head_plane = i0 + i * kPieces;
                if (head_plane >= 2 * p.cache.n_kv || !on)
                    continue;
                auto pair = [&](uint32_t f16) {
                    const float2 f = widen<__half>(f16);
                    return narrow_finite<T>(f.x * scale[i], f.y * scale[i]);
                };
                const int64_t plane = ((int64_t)(head_plane & 1) << p.cache.page_shift) * p.cache.n_kv * (2 * kVecs);
                store(out + plane + (head_plane >> 1) * (2 * kVecs), wide,
                      make_uint4(pair(e4m3_to_f16(x[i].x)), pair(e4m3_to_f16_high(x[i].x)), pair(e4m3_to_f16(x[i].y)),
                                 pair(e4m3_to_f16_high(x[i].y))),
                      make_uint4(pair(e4m3_to_f16(x[i].z)), pair(e4m3_to_f16_high(x[i].z)), pair(e4m3_to_f16(x[i].w)),
                                 pair(e4m3_to_f16_high(x[i].w))));
            }
        }
    }
}

template <typename T, int D>
cudaError_t launch(const Kv8Read &p, int sm_count, cudaStream_t s)
{
    const int64_t units = (int64_t)p.batch * groups_of(p.max_kv), most = (int64_t)sm_count * 8;
    // as many vectors of a thread in flight as a group has for it
    const int pieces = 2 * p.cache.n_kv * kGroup * (D / 16) / kThreads;
    return launch_pdl(pieces > 4 ? kv8_read_kernel<T, D, 8> : pieces > 2 ? kv8_read_kernel<T, D, 4> : kv8_read_kernel<T, D, 2>,
                      dim3((unsigned)(units < most ? units : most)), dim3(kThreads), 0, s, p);
}

}  // namespace

cudaError_t launch_kv8_read(const Kv8Read &p, int d, int dtype, int sm_count, cudaStream_t s)
{
    if (dtype == HS_FP16)
        return (d == 128 ? launch<__half, 128> : launch<__half, 64>)(p, sm_count, s);
    return (d == 128 ? launch<__nv_bfloat16, 128> : launch<__nv_bfloat16, 64>)(p, sm_count, s);
}

}  // namespace hs
