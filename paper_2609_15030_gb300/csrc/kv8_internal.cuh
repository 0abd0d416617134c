// Declarations and device steps shared by the calls of hs_kv8.h (kv8_api.cu) and their kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_internal.cuh"
#include "hs_kv8.h"

namespace hs {

// A model's positions as the kernels take them: pair i turns by turns[i] 2^-64 of a full turn for each
// position, so that a position's angle is an integer product modulo 2^64, without loss at any position.
struct RopeParams {
    uint64_t turns[HS_ROPE_MAX_PAIRS];
    double amplitude;
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
    int32_t window;               // rows whose groups a block begins
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

// The pairs of a lane's vectors as floats, x and y of pair j, and back into the vectors' order.
template <typename T>
__device__ __forceinline__ void pairs_of(const uint4 &a, const uint4 &b, bool half, float (&x)[8],
                                         float (&y)[8])
{
    const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 f = widen<T>(u[j]);
        if (half) {
            (j < 4 ? x : y)[2 * (j & 3)] = f.x;
            (j < 4 ? x : y)[2 * (j & 3) + 1] = f.y;
        } else {
            x[j] = f.x;
            y[j] = f.y;
        }
    }
}

template <typename T>
__device__ __forceinline__ void vectors_of(const float (&x)[8], const float (&y)[8], bool half, uint4 &a,
                                           uint4 &b)
{
    uint32_t u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        u[j] = half ? narrow<T>((j < 4 ? x : y)[2 * (j & 3)], (j < 4 ? x : y)[2 * (j & 3) + 1])
                    : narrow<T>(x[j], y[j]);
    a = make_uint4(u[0], u[1], u[2], u[3]);
    b = make_uint4(u[4], u[5], u[6], u[7]);
}

__device__ __forceinline__ void turn(float &x, float &y, float2 cs)
{
    const float t = x * cs.x - y * cs.y;
    y = y * cs.x + x * cs.y;
    x = t;
}

}  // namespace kv8
}  // namespace hs
