// Rotary positions: the rows of q and k turned by their positions (the recomputed suffix continues at its
// absolute positions, Section 2.2 of the paper).
//
// Pair (x, y) of a head becomes (x c - y s, y c + x s) with c, s = cos, sin of pos theta_i.  An angle is one
// 64-bit integer product modulo a full turn (RopeParams), off by |pos| 2^-65 turns at most, where pos theta_i in
// float32 is off by whole radians from some 10^7 on; its upper 32 bits go through one sine and cosine.
//
// A lane holds 8 pairs of a head: two 16-byte vectors, a head's halves or neighbours by the layout.  It computes
// their 8 sines and cosines once and takes them through several heads of the row.
#include "kv8_internal.cuh"

namespace hs {
namespace {

using namespace kv8;

constexpr int kThreads = 256;

template <typename T, int D, bool kHalf>
__global__ void __launch_bounds__(kThreads)
rope_kernel(const __grid_constant__ RopeRows p, const __grid_constant__ RopeParams rope)
{
    pdl_wait_and_release();
    turn_rows<T, D, kHalf>(p, rope, nullptr, (int64_t)blockIdx.x * (kThreads / (D / 16)));
}

template <typename T, int D>
cudaError_t launch(RopeRows r, const RopeParams &rope, int sm_count, cudaStream_t s)
{
    constexpr int kJobs = kThreads / (D / 16);
    r.slices = rope_slices(r.n_rows, r.n_heads + r.n_kv, sm_count, kJobs);
    const int64_t grid = (r.n_rows * r.slices + kJobs - 1) / kJobs;
    if (grid > INT32_MAX)
        return cudaErrorInvalidValue;
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
