// Softmax attention over the paged cache (full-attention layers): one warp per (row, head).
//
// With s_j = scale * log2(e) * q . k_j a row keeps m = max s_j, l = sum 2^(s_j - m) and
// a = sum 2^(s_j - m) v_j over the keys so far, float32, rescaled by 2^(m_old - m_new) when a
// larger score comes; o = a / l, lse = ln 2 * (m + log2 l).  Four keys at a time: their loads are
// independent, each lane holding D / 32 elements of a row.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_internal.cuh"

namespace hs {
namespace {

constexpr int kWarps = 4;
constexpr float kLn2 = 0.6931471805599453f;

template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
    using type = __nv_bfloat162;
};
template <>
struct Pair<__half> {
    using type = __half2;
};
__device__ __forceinline__ float2 widen(__nv_bfloat162 x) { return __bfloat1622float2(x); }
__device__ __forceinline__ float2 widen(__half2 x) { return __half22float2(x); }
template <typename T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16(x); }
template <>
__device__ __forceinline__ __half narrow<__half>(float x) { return __float2half(x); }

template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32)
attn_kernel(const __grid_constant__ AttnParams p)
{
    using T2 = typename Pair<T>::type;
    constexpr int E = D / 32;      // elements of a row per lane
    pdl_wait_and_release();
    const int b = blockIdx.y;
    const int lane = threadIdx.x & 31;
    const bool decode = p.kv_len != nullptr;
    const int64_t n = (decode ? 1 : (int64_t)p.n_tokens[b]) * p.n_heads;
    const int64_t page_mask = ((int64_t)1 << p.page_shift) - 1;
    int own = 0;
    if (decode) {
        own = p.kv_len[b];
        if (own < 0 || own > p.max_kv) {
            if (blockIdx.x == 0 && threadIdx.x == 0)
                report(p.d_err, HS_DEVERR_LENGTH);
            return;
        }
    }
    for (int64_t u = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); u < n;
         u += (int64_t)gridDim.x * kWarps) {
        const int t = (int)(u / p.n_heads), h = (int)(u - (int64_t)t * p.n_heads);
        const int kvh = h / p.group;
        const int64_t row = decode ? b : (int64_t)p.row0[b] + t;
        const int64_t keys = decode ? (int64_t)p.prefix_len + own : (int64_t)p.pos0[b] + t + 1;
        const T *q = static_cast<const T *>(p.q) + row * p.q_stride + h * D + lane * E;
        float qv[E], acc[E];
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 w = widen(*reinterpret_cast<const T2 *>(q + e));
            qv[e] = w.x, qv[e + 1] = w.y;
            acc[e] = acc[e + 1] = 0.f;
        }
        float m = -INFINITY, l = 0.f;
        for (int64_t j0 = 0; j0 < keys; j0 += 4) {
            const T *kp[4];
            bool ok[4];
            float s[4], vv[4][E];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int64_t j = j0 + x;
                ok[x] = j < keys;
                kp[x] = nullptr;
                if (!ok[x])
                    continue;
                const bool pre = j < p.prefix_len;
                const int64_t jj = pre ? j : j - p.prefix_len;
                const int32_t blk = pre ? p.prefix_table[jj >> p.page_shift]
                                        : p.table[b * p.max_pages + (jj >> p.page_shift)];
                if (blk < 0 || blk >= p.num_blocks) {
                    if (lane == 0)
                        report(p.d_err, HS_DEVERR_BLOCK_OOB);
                    continue;
                }
                kp[x] = static_cast<const T *>(p.cache) +
                        ((((int64_t)blk * 2 << p.page_shift) + (jj & page_mask)) * p.n_kv + kvh) * D +
                        lane * E;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                s[x] = 0.f;
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    float2 k2 = make_float2(0.f, 0.f), v2 = k2;
                    if (kp[x] != nullptr) {
                        k2 = widen(*reinterpret_cast<const T2 *>(kp[x] + e));
                        v2 = widen(*reinterpret_cast<const T2 *>(
                            kp[x] + ((int64_t)p.n_kv * D << p.page_shift) + e));
                    }
                    s[x] = fmaf(qv[e], k2.x, fmaf(qv[e + 1], k2.y, s[x]));
                    vv[x][e] = v2.x, vv[x][e + 1] = v2.y;
                }
            }
            float top = m;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
#pragma unroll
                for (int w = 16; w > 0; w >>= 1)
                    s[x] += __shfl_xor_sync(0xffffffffu, s[x], w);
                s[x] = ok[x] ? s[x] * p.scale_log2 : -INFINITY;
                top = fmaxf(top, s[x]);
            }
            const float f = exp2f(m - top);
            m = top;
            l *= f;
#pragma unroll
            for (int e = 0; e < E; ++e)
                acc[e] *= f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float w = exp2f(s[x] - m);
                l += w;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    acc[e] = fmaf(w, vv[x][e], acc[e]);
            }
        }
        const float inv = keys > 0 ? 1.f / l : 0.f;
        T *o = static_cast<T *>(p.o) + row * p.o_stride + h * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e)
            o[e] = narrow<T>(acc[e] * inv);
        if (p.lse != nullptr && lane == 0)
            p.lse[row * p.n_heads + h] = keys > 0 ? kLn2 * (m + log2f(l)) : -INFINITY;
    }
}

}  // namespace

cudaError_t launch_attn(const AttnParams &p, int d, int dtype, cudaStream_t s)
{
    int64_t most = 1;
    if (p.kv_len == nullptr)
        for (int b = 0; b < p.batch; ++b)
            most = p.n_tokens[b] > most ? p.n_tokens[b] : most;
    int64_t grid = (most * p.n_heads + kWarps - 1) / kWarps;
    if (grid > 65536)
        grid = 65536;
    const dim3 g((unsigned)grid, (unsigned)p.batch);
    if (dtype == HS_FP16)
        return d == 128 ? launch_pdl(attn_kernel<__half, 128>, g, dim3(kWarps * 32), 0, s, p)
                        : launch_pdl(attn_kernel<__half, 64>, g, dim3(kWarps * 32), 0, s, p);
    return d == 128 ? launch_pdl(attn_kernel<__nv_bfloat16, 128>, g, dim3(kWarps * 32), 0, s, p)
                    : launch_pdl(attn_kernel<__nv_bfloat16, 64>, g, dim3(kWarps * 32), 0, s, p);
}

}  // namespace hs
