// Declarations and device steps shared by the calls of hs_kv8.h (kv8_api.cu) and their kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_internal.cuh"
#include "hs_kv8.h"
#include "sm100_ptx.cuh"

namespace hs {

// A model's positions as the kernels take them: pair i turns by turns[i] 2^-64 + rest[i] 2^-96 of a full turn for each
// position, to half a unit.  So a position's angle is an integer product modulo 2^64, off by |pos| 2^-65 turns at most
// without the rest and by |pos| 2^-97 + 2^-64 with it.
struct RopeParams {
    uint64_t turns[HS_ROPE_MAX_PAIRS];
    int32_t rest[HS_ROPE_MAX_PAIRS];
    float gain, gain_low;         // the amplitude as a sum of two numbers
    int32_t pairs;                // dims / 2
    int32_t layout;
};

// q and k, or nullptr, in and out; strides in 16-byte vectors
struct RopeRows {
    const uint4 *q, *k;
    uint4 *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    const int64_t *pos;
    int64_t n_rows;
    int32_t n_heads, n_kv;        // 0 where the rows are left out
    int32_t slices;               // threads that share a row's heads
};

// the 8-bit cache
struct Kv8Cache {
    uint8_t *base;
    int64_t block_bytes;
    int64_t num_blocks;
    int32_t n_kv;
    int32_t page_shift;
};

// how a decode step is shared out
struct Kv8Plan {
    int32_t row_tiles;            // of a KV head's query rows
    int32_t items;                // of a request: row tiles of its KV heads
    int32_t warps, ctas;          // to a block; blocks
    int32_t per_row;              // warps that join a row
    Divisor by_row_tiles, by_items, by_warps, by_ctas;
};

struct Kv8Append {
    Kv8Cache cache;
    const uint4 *q, *k, *v;       // q: nullptr without positions
    uint4 *q_out;
    int64_t q_stride, kv_stride, q_out_stride;   // in 16-byte vectors
    const int64_t *pos, *slots;
    int64_t n_rows;
    int32_t *d_err;
    int32_t n_heads;
    int32_t windows;              // of 16 rows
    int32_t slices_log, parts_log;   // logarithms: teams that share a window's turned keys, warps for its other planes
    int32_t q_slices;             // threads that share a row's heads of q
    int32_t team_blocks, warp_blocks;   // in front of those for q
};

struct Kv8Read {
    Kv8Cache cache;
    const int32_t *table, *out_table, *kv_len;
    uint4 *out;
    int64_t out_blocks;
    int64_t max_pages;
    int32_t *d_err;
    int32_t batch;
    int32_t max_kv;
};

cudaError_t launch_rope(const RopeRows &r, const RopeParams &rope, int d, int dtype, int sm_count,
                        cudaStream_t s);
// rope: nullptr without positions
cudaError_t launch_kv8_append(Kv8Append a, const RopeParams *rope, int d, int dtype, int sm_count,
                              cudaStream_t s);
cudaError_t launch_kv8_read(const Kv8Read &r, int d, int dtype, int sm_count, cudaStream_t s);
// Fill in the schedule and say how many bytes of workspace it takes; -1: more units than 31 bits count.
int64_t plan_kv8_decode(AttnParams &p, Kv8Plan &plan, int d, int sm_count);
cudaError_t launch_kv8_decode(const AttnParams &p, const Kv8Plan &plan, const Kv8Cache &cache, int d, int dtype,
                              cudaStream_t s);

namespace kv8 {

constexpr int kGroup = HS_KV8_GROUP;

// ---- numbers -------------------------------------------------------------------------------

// two floats of a 16-bit pair and back (rounded to nearest, ties to even)
template <typename T>
__device__ __forceinline__ float2 widen(uint32_t x)
{
    if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value) {
        __half2 h;
        memcpy(&h, &x, 4);
        return __half22float2(h);
    } else {
        return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    }
}

template <typename T>
__device__ __forceinline__ uint32_t narrow(float lo, float hi)
{
    uint32_t x;
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 h = __floats2half2_rn(lo, hi);
        memcpy(&x, &h, 4);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        memcpy(&x, &h, 4);
    }
    return x;
}

// the same kept within the finite values of T; NaN stays
template <typename T>
__device__ __forceinline__ uint32_t narrow_finite(float lo, float hi)
{
    uint32_t x;
    if constexpr (std::is_same<T, __half>::value)
        asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(hi), "f"(lo));
    return x;
}

// two E4M3 numbers (the low 16 bits of x) as binary16, exact
__device__ __forceinline__ uint32_t e4m3_to_f16(uint32_t x)
{
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}"
        : "=r"(r) : "r"(x));
    return r;
}

// the same of the high 16 bits
__device__ __forceinline__ uint32_t e4m3_to_f16_high(uint32_t x)
{
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}"
        : "=r"(r) : "r"(x));
    return r;
}

// four floats as E4M3, x0 in the low byte: nearest, ties to even, NaN stays, beyond 448 is 448
__device__ __forceinline__ uint32_t to_e4m3(float x0, float x1, float x2, float x3)
{
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(r) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
    return r;
}

__device__ __forceinline__ float power_of_two(int e)     // -126 <= e <= 127
{
    return __int_as_float((e + 127) << 23);
}

// 2^-e of 2^e, -126 <= e <= 126
__device__ __forceinline__ float inverse(float power)
{
    return __uint_as_float(0x7f000000u - __float_as_uint(power));
}

// ---- addresses -----------------------------------------------------------------------------

// bytes of one (KV head, plane) of a block
template <int D>
__device__ __forceinline__ int64_t plane_bytes(const Kv8Cache &c)
{
    return (int64_t)D << c.page_shift;
}

// group g (counted over the cache) of a KV head's plane: its first byte, and its scale
template <int D>
__device__ __forceinline__ uint8_t *group_at(const Kv8Cache &c, int64_t blk, int in_page, int head_plane,
                                             float **scale)
{
    uint8_t *const at = c.base + blk * c.block_bytes;
    *scale = reinterpret_cast<float *>(at + 2 * c.n_kv * plane_bytes<D>(c)) +
             ((head_plane << (c.page_shift - 4)) + in_page);
    return at + head_plane * plane_bytes<D>(c) + (int64_t)in_page * (kGroup * D);
}

// ---- positions -----------------------------------------------------------------------------

// position times turns, as a signed fraction of a turn in units of 2^-64
__device__ __forceinline__ int64_t angle_of(uint64_t turns, int64_t pos)
{
    return (int64_t)(turns * (uint64_t)pos);
}

// the same with the rest
__device__ __forceinline__ int64_t angle_of(uint64_t turns, int32_t rest, int64_t pos)
{
    return angle_of(turns, pos) + __mul64hi(pos, (int64_t)rest * (1ll << 32));
}

// amplitude times (cos, sin) of an angle; its upper 32 bits are kept: 2^-32 of a turn
__device__ __forceinline__ float2 spin_of(int64_t angle, float amplitude)
{
    float s, c;
    sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, &s, &c);
    return make_float2(c * amplitude, s * amplitude);
}

// Where a lane's two 16-byte vectors of a head lie (D / 16 lanes to a head).  Lanes v < pairs / 8 hold the pairs
// 8 v to 8 v + 7, the others elements that are not turned.
__device__ __forceinline__ void lane_vectors(int v, int pairs, bool half, int &a, int &b)
{
    if (half && v < pairs / 8) {
        a = v;
        b = v + pairs / 8;
    } else {
        a = 2 * v;
        b = 2 * v + 1;
    }
}

// Eight pairs of a head as floats, two to a register pair: x[k] and y[k] of the pairs 2 k and 2 k + 1.
struct Pairs {
    uint64_t x[4], y[4];
};

// their cosines and sines
struct Spins {
    uint64_t c[4], s[4];
};

// a lane's vectors as pairs, and back
template <typename T, bool kHalf>
__device__ __forceinline__ Pairs pairs_of(const uint4 &a, const uint4 &b)
{
    const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    Pairs p;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = widen<T>(u[kHalf ? k : 2 * k]), g = widen<T>(u[kHalf ? k + 4 : 2 * k + 1]);
        p.x[k] = kHalf ? ptx::pair(f.x, f.y) : ptx::pair(f.x, g.x);
        p.y[k] = kHalf ? ptx::pair(g.x, g.y) : ptx::pair(f.y, g.y);
    }
    return p;
}

template <typename T, bool kHalf>
__device__ __forceinline__ void vectors_of(const Pairs &p, uint4 &a, uint4 &b)
{
    uint32_t u[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 x = ptx::unpair(p.x[k]), y = ptx::unpair(p.y[k]);
        u[kHalf ? k : 2 * k] = kHalf ? narrow<T>(x.x, x.y) : narrow<T>(x.x, y.x);
        u[kHalf ? k + 4 : 2 * k + 1] = kHalf ? narrow<T>(y.x, y.y) : narrow<T>(x.y, y.y);
    }
    a = make_uint4(u[0], u[1], u[2], u[3]);
    b = make_uint4(u[4], u[5], u[6], u[7]);
}

// (x, y) to (x c - y s, y c + x s)
__device__ __forceinline__ void turn(Pairs &p, const Spins &by)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t x = p.x[k], y = p.y[k];
        p.x[k] = ptx::fma2(y, by.s[k] ^ 0x8000000080000000ull, ptx::mul2(x, by.c[k]));
        p.y[k] = ptx::fma2(x, by.s[k], ptx::mul2(y, by.c[k]));
    }
}

// threads that share a row's heads: as many heads to a thread as fill the SMs; `jobs`: rows of a block at one slice
inline int32_t rope_slices(int64_t n_rows, int heads, int sm_count, int jobs)
{
    int64_t slices = 4;
    while (slices < heads && n_rows * slices < (int64_t)sm_count * 4 * jobs)
        slices *= 2;
    return (int32_t)(slices < heads ? slices : heads);
}

// Rows turned: every D / 16 lanes take a job, a row's heads slice, slice + slices, ...; the block's jobs begin at `job0`.  A
// lane's 8 sines and cosines serve all its heads, several of which are in flight.  Rows with a negative slot are
// left out (slots: nullptr, or of the rows).
template <typename T, int D, bool kHalf>
__device__ __forceinline__ void turn_rows(const RopeRows &p, const RopeParams &rope, const int64_t *slots, int64_t job0)
{
    constexpr int kLanes = D / 16, kAhead = 4;
    const int v = threadIdx.x % kLanes, heads = p.n_heads + p.n_kv;
    const bool turned = v < rope.pairs / 8;
    int a, b;
    lane_vectors(v, rope.pairs, kHalf, a, b);
    const int64_t job = job0 + threadIdx.x / kLanes, row = job / p.slices;
    const int slice = (int)(job - row * p.slices);
    if (row >= p.n_rows)
        return;
    const int64_t pos = turned ? __ldg(p.pos + row) : 0;
    if (slots != nullptr && __ldg(slots + row) < 0)
        return;
    Spins spins;
    for (int h0 = slice; h0 < heads; h0 += p.slices * kAhead) {
        uint4 in[kAhead][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * p.slices;
            if (h >= heads)
                break;
            const uint4 *const from = h < p.n_heads ? p.q + row * p.q_stride + h * (D / 8)
                                                    : p.k + row * p.k_stride + (h - p.n_heads) * (D / 8);
            in[i][0] = __ldcs(from + a);
            in[i][1] = __ldcs(from + b);
        }
        if (h0 == slice && turned) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = spin_of(angle_of(rope.turns[8 * v + 2 * k], pos), rope.gain),
                             g = spin_of(angle_of(rope.turns[8 * v + 2 * k + 1], pos), rope.gain);
                spins.c[k] = ptx::pair(f.x, g.x);
                spins.s[k] = ptx::pair(f.y, g.y);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * p.slices;
            if (h >= heads)
                break;
            if (turned) {
                Pairs x = pairs_of<T, kHalf>(in[i][0], in[i][1]);
                turn(x, spins);
                vectors_of<T, kHalf>(x, in[i][0], in[i][1]);
            }
            uint4 *const to = h < p.n_heads ? p.q_out + row * p.q_out_stride + h * (D / 8)
                                            : p.k_out + row * p.k_out_stride + (h - p.n_heads) * (D / 8);
            to[a] = in[i][0];
            to[b] = in[i][1];
        }
    }
}

}  // namespace kv8
}  // namespace hs
