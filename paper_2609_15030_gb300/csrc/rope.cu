// Rotary positions: the rows of q and k turned by their positions (the recomputed suffix continues at its
// absolute positions, Section 2.2 of the paper).
//
// Pair (x, y) of a head becomes (x c - y s, y c + x s) with c, s = cos, sin of pos theta_i.  An angle is one
// 64-bit integer product modulo a full turn (RopeParams), so nothing is lost at far positions, where
// pos theta_i in float32 is off by whole radians; its upper 32 bits go through one sine and cosine.
//
// A lane holds 8 pairs of a head: two 16-byte vectors, a head's halves or neighbours by the layout.  It computes
// their 8 sines and cosines once and takes them through several heads of the row.
#include "kv8_internal.cuh"

namespace hs {
namespace {

using namespace kv8;

constexpr int kThreads = 256;
constexpr int kAhead = 4;                    // heads of a lane in flight

template <typename T, int D, bool kHalf>
__global__ void __launch_bounds__(kThreads)
rope_kernel(const __grid_constant__ RopeRows p, const __grid_constant__ RopeParams rope)
{
    constexpr int kLanes = D / 16;
    pdl_wait_and_release();
    const int v = threadIdx.x % kLanes, heads = p.n_heads + p.n_kv;
    const bool turned = v < rope.pairs / 8;
    int a, b;
    lane_vectors(v, rope.pairs, kHalf, a, b);
    const int64_t jobs = p.n_rows * p.slices;
    for (int64_t job = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes; job < jobs;
         job += (int64_t)gridDim.x * (kThreads / kLanes)) {
        const int64_t row = job / p.slices;
        const int slice = (int)(job - row * p.slices);
        float2 cs[8];
        if (turned) {
            const int64_t pos = __ldg(p.pos + row);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                cs[j] = spin_of(angle_of(rope.turns[8 * v + j], pos), (float)rope.amplitude);
        }
        for (int h0 = slice; h0 < heads; h0 += p.slices * kAhead) {
            uint4 in[kAhead][2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int h = h0 + i * p.slices;
                if (h >= heads)
                    break;
                const uint4 *const from = h < p.n_heads
                                              ? p.q + row * p.q_stride + h * (D / 8)
                                              : p.k + row * p.k_stride + (h - p.n_heads) * (D / 8);
                in[i][0] = __ldcs(from + a);
                in[i][1] = __ldcs(from + b);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int h = h0 + i * p.slices;
                if (h >= heads)
                    break;
                if (turned) {
                    float x[8], y[8];
                    pairs_of<T>(in[i][0], in[i][1], kHalf, x, y);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        turn(x[j], y[j], cs[j]);
                    vectors_of<T>(x, y, kHalf, in[i][0], in[i][1]);
                }
                uint4 *const to = h < p.n_heads
                                      ? p.q_out + row * p.q_out_stride + h * (D / 8)
                                      : p.k_out + row * p.k_out_stride + (h - p.n_heads) * (D / 8);
                to[a] = in[i][0];
                to[b] = in[i][1];
            }
        }
    }
}

template <typename T, int D>
cudaError_t launch(RopeRows r, const RopeParams &rope, int sm_count, cudaStream_t s)
{
    constexpr int kPerBlock = kThreads / (D / 16);
    const int heads = r.n_heads + r.n_kv;
    // as many heads to a lane as fill the SMs
    int64_t slices = 4;
    while (slices < heads && r.n_rows * slices < (int64_t)sm_count * 4 * kPerBlock)
        slices *= 2;
    r.slices = (int32_t)(slices < heads ? slices : heads);
    int64_t grid = (r.n_rows * r.slices + kPerBlock - 1) / kPerBlock;
    if (grid > INT32_MAX)
        grid = INT32_MAX;
    return launch_pdl(rope.layout == HS_ROPE_HALF ? rope_kernel<T, D, true> : rope_kernel<T, D, false>,
                      dim3((unsigned)grid), dim3(kThreads), 0, s, r, rope);
}

}  // namespace

cudaError_t launch_rope(const RopeRows &r, const RopeParams &rope, int d, int dtype, int sm_count,
                        cudaStream_t s)
{
    if (dtype == HS_FP16)
        return (d == 128 ? launch<__half, 128> : launch<__half, 64>)(r, rope, sm_count, s);
    return (d == 128 ? launch<__nv_bfloat16, 128> : launch<__nv_bfloat16, 64>)(r, rope, sm_count, s);
}

}  // namespace hs
