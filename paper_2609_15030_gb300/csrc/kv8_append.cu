// New tokens' K and V rows of one layer quantised into their 8-bit pages, alone or with rotary positions on
// the way (the FP8 KV setting, Table 1 of the paper).
//
// Of a group of 16 tokens, KV head and plane: M = max |x| of the new values, need = the smallest
// 2^e >= M / 448, scale = need (a group that begins) or max(scale, need) (one that goes on; where it grows, the
// bytes that the group holds are rounded to the new scale), bytes = E4M3(x / scale).  With powers of two
// both divisions are exact, so each value is rounded once for each scale that it lives under.
//
// The rows of a group stand one behind the other: its first row's place (the row in front has another group)
// says who owns it.  A block takes a window of rows and the groups that begin in it; a warp takes one (KV
// head, plane) of these groups one after the other, 16 rows in registers (D / 16 lanes to a row,
// two 16-byte vectors each), so that M and the bytes come from one read.  Sines and cosines of the
// block's rows are computed once, in shared memory, for all heads.
#include "kv8_internal.cuh"

namespace hs {
namespace {

using namespace kv8;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kWindow = 16;                        // rows of a window at most
constexpr int kRows = 2 * kWindow - 1;             // rows that a window's groups may reach

// The largest magnitude of the turned keys of a lane's rows in float64, for one that lies next to a border between two scales.
template <typename T, int D, bool kHalf>
__device__ __noinline__ double largest_exact(const RopeParams &rope, const int64_t *pos, const uint4 *k,
                                             int64_t stride, int n, int v, int sub)
{
    double top = 0.0;
    int a, b;
    lane_vectors(v, rope.pairs, kHalf, a, b);
    for (int i = sub; i < n; i += 512 / D) {
        float x[8], y[8];
        pairs_of<T>(k[i * stride + a], k[i * stride + b], kHalf, x, y);
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
            double s = 0.0, c = 1.0;
            if (v < rope.pairs / 8) {
                sincospi((double)angle_of(rope.turns[8 * v + j], pos[i]) * 0x1p-63, &s, &c);
                s *= rope.amplitude;
                c *= rope.amplitude;
            }
            top = fmax(top, fmax(fabs(x[j] * c - y[j] * s), fabs(y[j] * c + x[j] * s)));
        }
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1)
        top = fmax(top, __shfl_xor_sync(0xffffffffu, top, w));
    return top;
}

template <typename T, int D, bool kRope, bool kHalf>
__global__ void __launch_bounds__(kThreads)
kv8_append_kernel(const __grid_constant__ Kv8Append p, const __grid_constant__ RopeParams rope)
{
    constexpr int kLanes = D / 16;                 // lanes to a row
    constexpr int kAtOnce = 32 / kLanes;           // rows of a warp at a time
    constexpr int kSteps = kGroup / kAtOnce;
    __shared__ float2 spins[kRope ? kRows : 1][D / 2];
    pdl_wait_and_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int v = lane % kLanes, sub = lane / kLanes;
    const int64_t r0 = (int64_t)blockIdx.x * p.window;

    // lane l: the slot and group of row r0 - 1 + l; the rows where a group of this window begins
    const int64_t mine = r0 - 1 + lane;
    const int64_t slot = mine >= 0 && mine < p.n_rows ? __ldg(p.slots + mine) : -1;
    const bool far = slot >= p.cache.num_blocks << p.cache.page_shift;
    if (far && warp == 0 && blockIdx.y == 0 && lane > 0)
        report(p.d_err, HS_DEVERR_BLOCK_OOB);
    const int64_t group = slot < 0 || far ? -1 : slot / kGroup;
    const int64_t before = __shfl_up_sync(0xffffffffu, group, 1);
    const unsigned begins = __ballot_sync(0xffffffffu, lane >= 1 && lane <= p.window && group >= 0 &&
                                                           group != before);
    // rows of the group that begins with lane l's row
    auto rows_from = [&](int l) {
        const unsigned other = ~(__ballot_sync(0xffffffffu, group == __shfl_sync(0xffffffffu, group, l)) >> l);
        const int n = __ffs(other) - 1;
        return n < 0 || n > kGroup ? kGroup : n;
    };

    if constexpr (kRope) {
        int rows = p.window;
        if (begins != 0) {
            const int last = 31 - __clz(begins), end = last - 1 + rows_from(last);
            rows = end > rows ? end : rows;
        }
        if (r0 + rows > p.n_rows)
            rows = (int)(p.n_rows - r0);
        for (int i = threadIdx.x; i < rows * rope.pairs; i += kThreads) {
            const int r = i / rope.pairs, j = i - r * rope.pairs;
            spins[r][j] = spin_of(angle_of(rope.turns[j], __ldg(p.pos + r0 + r)), (float)rope.amplitude);
        }
        __syncthreads();
    }

    // K and V
    const bool turned = kRope && v < rope.pairs / 8;
    for (int job = warp + kWarps * blockIdx.y; job < 2 * p.cache.n_kv; job += kWarps * gridDim.y) {
        const int head = job >> 1, plane = job & 1;
        const bool turns = turned && plane == 0;
        const bool half = kRope && kHalf && plane == 0;
        int a, b;
        lane_vectors(v, kRope ? rope.pairs : 0, half, a, b);
        for (unsigned left = begins; left != 0; left &= left - 1) {
            const int l = __ffs(left) - 1, n = rows_from(l);
            const int64_t row = r0 - 1 + l;
            const int64_t g = __shfl_sync(0xffffffffu, group, l);
            const int shift = p.cache.page_shift - 4;
            float *scale_at;
            uint8_t *const at = group_at<D>(p.cache, g >> shift, (int)(g & (((int64_t)1 << shift) - 1)), job,
                                            &scale_at);
            const float old = *scale_at;
            const uint4 *const from = (plane ? p.v : p.k) + row * p.kv_stride + head * (D / 8);
            uint4 in[kSteps][2];
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int i = s * kAtOnce + sub;
                in[s][0] = in[s][1] = make_uint4(0, 0, 0, 0);
                if (i < n) {
                    in[s][0] = __ldcs(from + i * p.kv_stride + a);
                    in[s][1] = __ldcs(from + i * p.kv_stride + b);
                }
            }
            // the values of step s
            auto values = [&](int s, float (&x)[8], float (&y)[8]) {
                pairs_of<T>(in[s][0], in[s][1], half, x, y);
                if (turns) {
                    const int i = s * kAtOnce + sub;
                    const float2 *const cs = spins[l - 1 + (i < n ? i : 0)] + 8 * v;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        turn(x[j], y[j], cs[j]);
                }
            };
            float top = 0.f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                float x[8], y[8];
                values(s, x, y);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    top = fmaxf(top, fmaxf(fabsf(x[j]), fabsf(y[j])));
            }
            uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
            const bool odd = bits >= 0x7f800000u;       // an infinity among the values
            if (odd) {
                top = 0.f;
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    float x[8], y[8];
                    values(s, x, y);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        top = fabsf(x[j]) < INFINITY ? fmaxf(top, fabsf(x[j])) : top;
                        top = fabsf(y[j]) < INFINITY ? fmaxf(top, fabsf(y[j])) : top;
                    }
                }
                bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
            }
            // 448 = 1.75 2^8
            int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
            if (kRope && plane == 0 && !odd && abs((int)(bits & 0x7fffffu) - 0x600000) <= 8) {
                const double t = largest_exact<T, D, kHalf>(rope, p.pos + row, from, p.kv_stride, n, v, sub);
                const int64_t w = __double_as_longlong(t);
                e = (int)(w >> 52) - 1023 - 8 + ((w & 0xfffffffffffffll) > 0xc000000000000ll);
            }
            const float need = power_of_two(e < -126 ? -126 : e);
            const int spot = (int)(__shfl_sync(0xffffffffu, slot, (l + lane) & 31) & (kGroup - 1));
            const unsigned tokens = __reduce_or_sync(0xffffffffu, lane < n ? 1u << spot : 0u);
            const bool anew = tokens & 1;
            const float scale = anew ? need : fmaxf(old, need);
            if (!anew && need > old) {
                // what the group holds, 16 bytes to a lane
                const float shrink = old / need;
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int i = s * kAtOnce + sub;
                    if ((tokens >> i) & 1)
                        continue;
                    uint4 *const w = reinterpret_cast<uint4 *>(at + i * D) + v;
                    const uint4 y = *w;
                    auto again = [&](uint32_t u) {
                        const float2 f = widen<__half>(e4m3_to_f16(u)), h = widen<__half>(e4m3_to_f16_high(u));
                        return to_e4m3(f.x * shrink, f.y * shrink, h.x * shrink, h.y * shrink);
                    };
                    *w = make_uint4(again(y.x), again(y.y), again(y.z), again(y.w));
                }
            }
            const float by = 1.f / scale;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int i = s * kAtOnce + sub;
                const int token = __shfl_sync(0xffffffffu, spot, i);
                if (i >= n)
                    continue;
                float x[8], y[8];
                values(s, x, y);
                if (odd) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[j] = fabsf(x[j]) < INFINITY ? x[j] : NAN;
                        y[j] = fabsf(y[j]) < INFINITY ? y[j] : NAN;
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] *= by;
                    y[j] *= by;
                }
                uint8_t *const to = at + token * D;
                if (half && turned) {
                    *reinterpret_cast<uint2 *>(to + 8 * a) =
                        make_uint2(to_e4m3(x[0], x[1], x[2], x[3]), to_e4m3(x[4], x[5], x[6], x[7]));
                    *reinterpret_cast<uint2 *>(to + 8 * b) =
                        make_uint2(to_e4m3(y[0], y[1], y[2], y[3]), to_e4m3(y[4], y[5], y[6], y[7]));
                } else if (half) {              // x and y hold the two vectors one behind the other
                    *reinterpret_cast<uint4 *>(to + 8 * a) =
                        make_uint4(to_e4m3(x[0], x[1], x[2], x[3]), to_e4m3(x[4], x[5], x[6], x[7]),
                                   to_e4m3(y[0], y[1], y[2], y[3]), to_e4m3(y[4], y[5], y[6], y[7]));
                } else {                        // and here every other element
                    *reinterpret_cast<uint4 *>(to + 8 * a) =
                        make_uint4(to_e4m3(x[0], y[0], x[1], y[1]), to_e4m3(x[2], y[2], x[3], y[3]),
                                   to_e4m3(x[4], y[4], x[5], y[5]), to_e4m3(x[6], y[6], x[7], y[7]));
                }
            }
            if (lane == 0)
                *scale_at = scale;
        }
    }

    // q
    if constexpr (kRope) {
        if (p.q == nullptr)
            return;
        int a, b;
        lane_vectors(v, rope.pairs, kHalf, a, b);
        const int each = kThreads / kLanes;
        for (int i = threadIdx.x / kLanes + each * blockIdx.y; i < p.window * p.n_heads; i += each * gridDim.y) {
            const int r = i / p.n_heads, h = i - r * p.n_heads;
            const int64_t row = r0 + r;
            if (row >= p.n_rows || __ldg(p.slots + row) < 0)
                continue;
            const uint4 *const from = p.q + row * p.q_stride + h * (D / 8);
            uint4 *const to = p.q_out + row * p.q_out_stride + h * (D / 8);
            uint4 y0 = __ldcs(from + a), y1 = __ldcs(from + b);
            if (turned) {
                float x[8], y[8];
                pairs_of<T>(y0, y1, kHalf, x, y);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    turn(x[j], y[j], spins[r][8 * v + j]);
                vectors_of<T>(x, y, kHalf, y0, y1);
            }
            to[a] = y0;
            to[b] = y1;
        }
    }
}

template <typename T, int D>
cudaError_t launch(Kv8Append p, const RopeParams *rope, int sm_count, cudaStream_t s)
{
    // windows of one row where there are few, up to 16 rows where those fill the SMs
    p.window = 1;
    while (p.window < kWindow && p.n_rows >= (int64_t)sm_count * 2 * p.window)
        p.window *= 2;
    const int64_t grid = (p.n_rows + p.window - 1) / p.window;
    if (grid > INT32_MAX)
        return cudaErrorInvalidValue;
    const int jobs = 2 * p.cache.n_kv + (rope != nullptr && p.q != nullptr ? p.n_heads : 0);
    int y = (int)((2 * sm_count + grid - 1) / grid);
    if (y > (jobs + kWarps - 1) / kWarps)
        y = (jobs + kWarps - 1) / kWarps;
    const dim3 blocks((unsigned)grid, (unsigned)y);
    if (rope == nullptr)
        return launch_pdl(kv8_append_kernel<T, D, false, false>, blocks, dim3(kThreads), 0, s, p,
                          RopeParams{});
    return launch_pdl(rope->layout == HS_ROPE_HALF ? kv8_append_kernel<T, D, true, true>
                                                   : kv8_append_kernel<T, D, true, false>,
                      blocks, dim3(kThreads), 0, s, p, *rope);
}

}  // namespace

cudaError_t launch_kv8_append(Kv8Append p, const RopeParams *rope, int d, int dtype, int sm_count,
                              cudaStream_t s)
{
    if (dtype == HS_FP16)
        return (d == 128 ? launch<__half, 128> : launch<__half, 64>)(p, rope, sm_count, s);
    return (d == 128 ? launch<__nv_bfloat16, 128> : launch<__nv_bfloat16, 64>)(p, rope, sm_count, s);
}

}  // namespace hs
