// The shares of a call whose requests' lengths lie on the device: units of 16 tokens, counted over the requests.
#pragma once

#include "attn_walk.cuh"
#include "kv8_internal.cuh"

namespace hs {
namespace kv8 {

// the units in front of each request, and its length (-1: out of bounds, it has no units)
struct Lengths {
    int32_t len[HS_MAX_BATCH];
    int32_t before[HS_MAX_BATCH + 1];
};

// Filled in by a block's first warp; every thread waits for it.  units(len): of a request.
template <typename Units>
__device__ __forceinline__ void read_lengths(Lengths &all, const int32_t *kv_len, int batch, int max_kv,
                                             int32_t *d_err, Units units)
{
    constexpr int kAhead = 4;                      // loads that do not wait for one another
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int sum = 0;
#pragma unroll 1
        for (int b0 = 0; b0 < batch; b0 += 32 * kAhead) {
            int n[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                n[i] = b0 + i * 32 + lane < batch ? kv_len[b0 + i * 32 + lane] : -1;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int b = b0 + i * 32 + lane;
                const bool fine = n[i] >= 0 && n[i] <= max_kv;
                if (!fine && b < batch && blockIdx.x == 0)
                    report(d_err, HS_DEVERR_LENGTH);
                const int x = fine ? units(n[i]) : 0;
                const int incl = attn::warp_scan(x, lane);
                if (b < batch) {
                    all.len[b] = fine ? n[i] : -1;
                    all.before[b] = sum + incl - x;
                }
                sum += __shfl_sync(0xffffffffu, incl, 31);
                if (b0 + i * 32 + 32 >= batch)
                    break;
            }
        }
        if (lane == 0)
            all.before[batch] = sum;
    }
    __syncthreads();
}

// the request with unit u, for a whole warp
__device__ __forceinline__ int request_of(const Lengths &all, int batch, int u, int lane)
{
    int b = 0;
    for (int b0 = 0; b0 < batch; b0 += 32) {
        const bool past = b0 + lane < batch && all.before[b0 + lane + 1] <= u;
        const unsigned m = __ballot_sync(0xffffffffu, past);
        b += __popc(m);
        if (m != 0xffffffffu)
            break;
    }
    return b;
}

// Units shared out evenly, the first shares with one more where that does not go up: the first unit of share i, and the
// share with unit u.
struct Shares {
    int each, more;
    // n units over by.d shares, or over n where these are fewer
    __device__ __forceinline__ Shares(int n, const Divisor &by) : each(by.div(n)), more(n - each * by.d) {}
    __device__ __forceinline__ int begin(int i) const
    {
        return i * each + min(i, more);
    }
    __device__ __forceinline__ int of(int u) const
    {
        return u < more * (each + 1) ? u / (each + 1) : more + (u - more * (each + 1)) / each;
    }
};

__host__ __device__ __forceinline__ int groups_of(int len)
{
    return (int)(((unsigned)len + kGroup - 1) / kGroup);
}

}  // namespace kv8
}  // namespace hs
