// One decode step over the 8-bit cache (the FP8 KV setting, Table 1 of the paper).
//
// Per query row, with s_j = scale log2(e) q . k_j:  m a number near max s_j, l = sum 2^(s_j - m),
// a = sum 2^(s_j - m) v_j in float32; o = a / l, lse = ln 2 (m + log2 l).  m follows the maximum when a tile
// exceeds it by more than 2^8.
//
// Bytes to numbers.  E4M3 lies within binary16, so keys and values become binary16 without loss on their way
// from the load to the tensor core.  A key's scale is a factor of its scores; a value's one goes into its
// weight, w_j = 2^(s_j - m) 2^(7 - E) scale_j with 2^E the largest scale so far, so that weights are at most 2^15 and one is
// rounded to nothing only below 2^-32 of the largest.  A bf16 q is scaled to binary16 by a power of two
// for each row.
//
// Shares.  A tile is a group of 16 tokens.  Every warp has a contiguous run of tiles of its own, shared out
// evenly over all warps of the GPU from the device lengths, with no hand-over until its end: a warp loads its keys and
// values into registers (they arrive in the order of the tensor core's operands, whose sums over d
// and tokens may go in any order), S^T = K Q^T (16 tokens x 8 rows for each instruction), turns the weights'
// tile by a matrix transpose between lanes, O^T += V^T W^T.  The warps of a block join their parts of an
// item (request, KV head, 8 or 16 query rows) in shared memory; an item with tiles in several blocks leaves a part
// for each in the workspace, and a second kernel joins these.  With `unsplit`, and where the bound is short,
// a block takes whole items instead.
//
// Few rows share a tile's bytes (the heads of one KV head), so the step is bound by HBM; products of M = 128 rows as in
// the 16-bit attention would leave most of the tensor core's rows empty and the bytes would have to
// become numbers on a way through shared memory.
#include "kv8_walk.cuh"

namespace hs {
namespace kv8 {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;

// floats of a part: per row m and l, then its sums, rows padded against bank conflicts
template <int D, int R>
constexpr int kPartFloats = 2 * R + R * (D + 4);

// one of a block's parts
struct Part {
    int32_t b, item;              // item: KV head * row tiles + row tile
    int32_t starts, ends;         // with the item's first and last tile
    int32_t used;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint4 load16(const void *p)
{
    uint4 x;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
    return x;
}

__device__ __forceinline__ uint2 load8(const void *p)
{
    uint2 x;
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "l"(p));
    return x;
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                    uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// an 8 x 8 matrix of 16-bit numbers, turned between lanes
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// items of a request, and the units of one
struct Shape {
    int row_tiles, per_request;
    __host__ __device__ Shape(const AttnParams &p, int rows)
        : row_tiles((p.group + rows - 1) / rows), per_request(row_tiles * p.n_kv)
    {
    }
    __host__ __device__ static int units(int len)
    {
        return len > 0 ? groups_of(len) : 1;      // an empty row is written by someone
    }
};

// where the results of an item's rows go
template <int R>
struct Rows {
    int b, head, n;               // head: of the first row
    __device__ Rows(const AttnParams &p, const Shape &shape, int b_, int item) : b(b_)
    {
        const int kvh = item / shape.row_tiles, rt = item - kvh * shape.row_tiles;
        head = kvh * p.group + rt * R;
        n = min(R, p.group - rt * R);
    }
};

// A warp's part of an item: NT tiles of 8 rows.  A lane (g = lane / 4, t = lane % 4) has the tokens g and g + 8 of
// scores and the columns [g D/8, (g + 1) D/8) of sums, of the rows 2 t and 2 t + 1 of each tile.
template <typename T, int D, int NT>
struct Warp {
    static constexpr int R = 8 * NT, C = D / 64;
    uint32_t q[C * 4][NT][2];
    float factor[NT][2];          // of scores, beside the keys' scale
    float m[NT][2], l[NT][2];
    float o[D / 16][NT][4];
    float top;                    // 2^E

    __device__ __forceinline__ void begin(const AttnParams &p, const Rows<R> &rows, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
        top = 0x1p-100f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool on = n * 8 + g < rows.n;
            const T *const row = static_cast<const T *>(p.q) + rows.b * p.q_stride +
                                 (int64_t)(rows.head + n * 8 + (on ? g : 0)) * D;
            uint32_t x[C][8];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint4 *const at = reinterpret_cast<const uint4 *>(row + c * 64 + t * 16);
                const uint4 y0 = at[0], y1 = at[1];
                x[c][0] = y0.x, x[c][1] = y0.y, x[c][2] = y0.z, x[c][3] = y0.w;
                x[c][4] = y1.x, x[c][5] = y1.y, x[c][6] = y1.z, x[c][7] = y1.w;
            }
            float by = p.scale_log2;
            if constexpr (!std::is_same<T, __half>::value) {
                float most = 0.f;
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 f = widen<T>(x[c][i]);
                        most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
                    }
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
                // the largest to [2^14, 2^15)
                int e = (int)(__float_as_uint(most) >> 23) - 127 - 14;
                e = e < -120 ? -120 : e > 113 ? 113 : e;
                const float down = power_of_two(-e);
                by *= power_of_two(e);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 f = widen<T>(x[c][i]);
                        x[c][i] = narrow<__half>(f.x * down, f.y * down);
                    }
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    q[c * 4 + i / 2][n][i & 1] = on ? x[c][i] : 0u;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                factor[n][i] = __shfl_sync(0xffffffffu, by, (2 * t + i) * 4);
                m[n][i] = -INFINITY;
                l[n][i] = 0.f;
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    o[d][n][i] = 0.f;
        }
    }

    // scores of a tile: k[c][i] the 16 bytes [64 c + 16 t, + 16) of token g + 8 i
    __device__ __forceinline__ void scores(const uint4 (&k)[C][2], float scale, float (&s)[NT][4]) const
    {
        float s2[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s[n][i] = s2[n][i] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const uint32_t x[4] = {k[c][0].x, k[c][0].y, k[c][0].z, k[c][0].w};
            const uint32_t y[4] = {k[c][1].x, k[c][1].y, k[c][1].z, k[c][1].w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t a0 = e4m3_to_f16(x[w]), a1 = e4m3_to_f16(y[w]), a2 = e4m3_to_f16_high(x[w]),
                               a3 = e4m3_to_f16_high(y[w]);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    mma((w & 1) ? s2[n] : s[n], a0, a1, a2, a3, q[c * 4 + w][n][0], q[c * 4 + w][n][1]);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // a product of both scales beyond float32 belongs to scores of 0, or to ones out of range
            const float f0 = fminf(factor[n][0] * scale, 3.4e38f), f1 = fminf(factor[n][1] * scale, 3.4e38f);
            s[n][0] = (s[n][0] + s2[n][0]) * f0;
            s[n][1] = (s[n][1] + s2[n][1]) * f1;
            s[n][2] = (s[n][2] + s2[n][2]) * f0;
            s[n][3] = (s[n][3] + s2[n][3]) * f1;
        }
    }

    // scores into weights, as the second product's operand
    __device__ __forceinline__ void weights(float (&s)[NT][4], float scale, uint32_t (&w)[NT][2])
    {
        bool more = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
            more = more || fmaxf(s[n][0], s[n][2]) > m[n][0] + 8.f || fmaxf(s[n][1], s[n][3]) > m[n][1] + 8.f;
        if (__any_sync(0xffffffffu, more)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float x = fmaxf(s[n][i], s[n][i + 2]);
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                    if (x > m[n][i]) {
                        const float h = ex2(m[n][i] - x);
                        m[n][i] = x;
                        l[n][i] *= h;
#pragma unroll
                        for (int d = 0; d < D / 16; ++d) {
                            o[d][n][i] *= h;
                            o[d][n][i + 2] *= h;
                        }
                    }
                }
        }
        if (scale > top) {
            // a power of two even where the cache's scale is none
            const float up = __uint_as_float(__float_as_uint(scale) & 0x7f800000u), h = top / up;
            top = up;
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        o[d][n][i] *= h;
        }
        const float by = scale * (128.f / top);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = ex2(s[n][i] - m[n][i & 1]);
                l[n][i & 1] += x[i];
            }
            w[n][0] = transposed(narrow<__half>(x[0] * by, x[1] * by));
            w[n][1] = transposed(narrow<__half>(x[2] * by, x[3] * by));
        }
    }

    // sums of a tile: v[i] the bytes [g D/8, + D/8) of the tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
    template <int N>
    __device__ __forceinline__ void sums(const uint32_t (&v)[4][N], const uint32_t (&w)[NT][2])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            // bytes of two tokens side by side
            const uint32_t x0 = __byte_perm(v[0][i], v[1][i], 0x5140), x1 = __byte_perm(v[0][i], v[1][i], 0x7362);
            const uint32_t y0 = __byte_perm(v[2][i], v[3][i], 0x5140), y1 = __byte_perm(v[2][i], v[3][i], 0x7362);
            const uint32_t a0 = e4m3_to_f16(x0), a1 = e4m3_to_f16_high(x0), a2 = e4m3_to_f16(y0),
                           a3 = e4m3_to_f16_high(y0);
            const uint32_t b0 = e4m3_to_f16(x1), b1 = e4m3_to_f16_high(x1), b2 = e4m3_to_f16(y1),
                           b3 = e4m3_to_f16_high(y1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                mma(o[2 * i][n], a0, a1, a2, a3, w[n][0], w[n][1]);
                mma(o[2 * i + 1][n], b0, b1, b2, b3, w[n][0], w[n][1]);
            }
        }
    }

    // the rows' l over all tokens
    __device__ __forceinline__ void end()
    {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], 4);
                l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], 8);
                l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], 16);
            }
    }

    // column j of a lane's D / 8, of row 2 t + i
    __device__ __forceinline__ float sum(int n, int i, int j) const
    {
        return o[j / 2][n][(j & 1) * 2 + i];
    }

    __device__ __forceinline__ void write(const AttnParams &p, const Rows<R> &rows, int lane) const
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = n * 8 + 2 * t + i;
                if (r >= rows.n)
                    continue;
                const float by = l[n][i] == 0.f ? 0.f : top * 0x1p-7f / l[n][i];
                uint32_t x[D / 16];
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
                    x[j] = narrow<T>(within<T>(sum(n, i, 2 * j) * by), within<T>(sum(n, i, 2 * j + 1) * by));
                uint4 *const to = reinterpret_cast<uint4 *>(static_cast<T *>(p.o) + rows.b * p.o_stride +
                                                            (int64_t)(rows.head + r) * D + g * (D / 8));
#pragma unroll
                for (int j = 0; j < D / 64; ++j)
                    to[j] = make_uint4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                if (p.lse != nullptr && g == 0)
                    p.lse[(int64_t)rows.b * p.n_heads + rows.head + r] =
                        l[n][i] == 0.f ? -INFINITY : 0.6931471805599453f * (m[n][i] + log2f(l[n][i]));
            }
    }

    __device__ __forceinline__ void leave(float *part, int lane) const
    {
        const int g = lane >> 2, t = lane & 3;
        const float by = top * 0x1p-7f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = n * 8 + 2 * t + i;
                if (g == 0) {
                    part[2 * r] = m[n][i];
                    part[2 * r + 1] = l[n][i];
                }
                float4 *const to = reinterpret_cast<float4 *>(part + 2 * R + r * (D + 4) + g * (D / 8));
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
                    to[j] = make_float4(sum(n, i, 4 * j) * by, sum(n, i, 4 * j + 1) * by,
                                        sum(n, i, 4 * j + 2) * by, sum(n, i, 4 * j + 3) * by);
            }
    }
};

// the tiles of one request's KV head, as a warp loads them
template <int D>
struct Tiles {
    const Kv8Cache &cache;
    const int32_t *table;         // the request's row
    int pages;                    // entries of it
    int head, lane, num_blocks;
    int32_t *d_err;
    int first;                    // page of ids' lane 0
    int32_t ids;                  // this lane's entry

    __device__ __forceinline__ void fetch(int page)
    {
        first = page;
        ids = page + lane < pages ? __ldg(table + page + lane) : 0;
        if (ids < 0 || ids >= cache.num_blocks) {
            report(d_err, HS_DEVERR_BLOCK_OOB);
            ids = -1;
        }
    }
    // the first byte of a tile's keys, nullptr where its page is none
    __device__ __forceinline__ const uint8_t *find(int tile, const float **scale)
    {
        const int shift = cache.page_shift - 4, page = tile >> shift;
        if (page - first >= 32)
            fetch(page);
        const int id = __shfl_sync(0xffffffffu, ids, page - first);
        if (id < 0)
            return nullptr;
        float *at;
        const uint8_t *const k = group_at<D>(cache, id, tile & ((1 << shift) - 1), 2 * head, &at);
        *scale = at;
        return k;
    }
};

template <typename T, int D, int NT>
__device__ __forceinline__ void walk(const AttnParams &p, const Kv8Cache &cache, Warp<T, D, NT> &w, int b, int len, int kvh,
                                     const Rows<8 * NT> &rows, int tile, int n, int lane)
{
    constexpr int C = D / 64;
    const int g = lane >> 2, t = lane & 3;
    Tiles<D> tiles{cache, p.table + (int64_t)b * p.max_pages, ((len - 1) >> cache.page_shift) + 1, kvh, lane, 0, p.d_err, 0, 0};
    if (n > 0)
        tiles.fetch(tile >> (cache.page_shift - 4));
    uint4 k[C][2];
    uint32_t v[4][D / 32];
    float k_scale = 0.f, v_scale = 0.f;
    const uint8_t *at = nullptr;
    const float *scale_at = nullptr;
    const int64_t plane = plane_bytes<D>(cache);
    const int groups = 1 << (cache.page_shift - 4);
    auto load_k = [&](int i) {
        at = tiles.find(i, &scale_at);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                k[c][j] = at != nullptr ? load16(at + (g + 8 * j) * D + c * 64 + t * 16) : make_uint4(0, 0, 0, 0);
        k_scale = at != nullptr ? __ldg(scale_at) : 0.f;
    };
    auto load_v = [&]() {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint8_t *const from = at + plane + (2 * t + (i & 1) + (i >> 1) * 8) * D + g * (D / 8);
            if constexpr (D == 128) {
                const uint4 x = at != nullptr ? load16(from) : make_uint4(0, 0, 0, 0);
                v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
            } else {
                const uint2 x = at != nullptr ? load8(from) : make_uint2(0, 0);
                v[i][0] = x.x, v[i][1] = x.y;
            }
        }
        v_scale = at != nullptr ? __ldg(scale_at + groups) : 0.f;
    };
    if (n > 0) {
        load_k(tile);
        load_v();
    }
    w.begin(p, rows, lane);
    for (int i = tile; i < tile + n; ++i) {
        float s[NT][4];
        uint32_t x[NT][2];
        w.scores(k, k_scale, s);
        if (i + 1 < tile + n)
            load_k(i + 1);
        const int left = len - i * kGroup;
        if (left < kGroup) {
            // behind the last key: no score, and values of zero (a weight of 0 times NaN is NaN)
#pragma unroll
            for (int a = 0; a < NT; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (g + 8 * (c >> 1) >= left)
                        s[a][c] = -INFINITY;
#pragma unroll
            for (int a = 0; a < 4; ++a)
                if (2 * t + (a & 1) + (a >> 1) * 8 >= left)
#pragma unroll
                    for (int c = 0; c < D / 32; ++c)
                        v[a][c] = 0;
        }
        w.weights(s, v_scale, x);
        w.sums(v, x);
        if (i + 1 < tile + n)
            load_v();
    }
    w.end();
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1)
kv8_decode_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ Kv8Cache cache)
{
    constexpr int R = 8 * NT, kSlots = 2 * kWarps;
    extern __shared__ float4 shared[];
    float *const parts = reinterpret_cast<float *>(shared);
    __shared__ Lengths all;
    __shared__ Part part[kSlots];
    pdl_wait_and_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Shape shape(p, R);
    read_lengths(all, p.kv_len, p.batch, p.max_kv, p.d_err,
                 [&](int len) { return Shape::units(len) * shape.per_request; });
    const int units = all.before[p.batch];

    // the block's run: its share of all units, or one whole item after the other
    for (int turn = blockIdx.x;; turn += gridDim.x) {
        int u0, u1, b = 0;
        if (p.unsplit) {
            if (turn >= p.batch * shape.per_request)
                return;
            b = turn / shape.per_request;
            if (all.len[b] < 0)
                continue;
            const int n = Shape::units(all.len[b]);
            u0 = all.before[b] + (turn - b * shape.per_request) * n;
            u1 = u0 + n;
        } else {
            u0 = attn::first_unit(units, gridDim.x, blockIdx.x);
            u1 = attn::first_unit(units, gridDim.x, blockIdx.x + 1);
        }
        if (threadIdx.x < kSlots)
            part[threadIdx.x].used = 0;
        __syncthreads();
        int u = u0 + (int)((int64_t)(u1 - u0) * warp / kWarps);
        const int end = u0 + (int)((int64_t)(u1 - u0) * (warp + 1) / kWarps);
        if (u < end) {
            b = request_of(all, p.batch, u, lane);
            int per = Shape::units(all.len[b]);
            int item = (u - all.before[b]) / per, tile = (u - all.before[b]) - item * per;
            int slot = 2 * warp;
            while (u < end) {
                const int len = all.len[b], n = min(per - tile, end - u);
                const Rows<R> rows(p, shape, b, item);
                Warp<T, D, NT> w;
                walk<T, D, NT>(p, cache, w, b, len, item / shape.row_tiles, rows, tile, len > 0 ? n : 0, lane);
                if (n == per) {
                    w.write(p, rows, lane);
                } else {
                    w.leave(parts + slot * kPartFloats<D, R>, lane);
                    if (lane == 0)
                        part[slot] = Part{b, item, tile == 0, tile + n == per, 1};
                    ++slot;
                }
                u += n;
                tile = 0;
                if (++item == shape.per_request && u < end) {
                    item = 0;
                    do
                        ++b;
                    while (all.before[b + 1] == all.before[b]);
                    per = Shape::units(all.len[b]);
                }
            }
        }
        __syncthreads();
        // join the parts of each item, which stand one behind the other
        for (int s0 = 0; s0 < kSlots;) {
            if (!part[s0].used) {
                ++s0;
                continue;
            }
            int s1 = s0, last = s0;
            for (; s1 < kSlots; ++s1)
                if (part[s1].used) {
                    if (part[s1].b != part[s0].b || part[s1].item != part[s0].item)
                        break;
                    last = s1;
                }
            const Rows<R> rows(p, shape, part[s0].b, part[s0].item);
            const bool whole = part[s0].starts && part[last].ends;
            float *const left = p.part + (int64_t)(2 * blockIdx.x + part[s0].starts) * kPartFloats<D, R>;
            for (int i = threadIdx.x; i < rows.n * (D / 4); i += kThreads) {
                const int r = i / (D / 4), c = i - r * (D / 4);
                float m = -INFINITY, l = 0.f;
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int s = s0; s < s1; ++s)
                    if (part[s].used)
                        m = fmaxf(m, parts[s * kPartFloats<D, R> + 2 * r]);
                for (int s = s0; s < s1; ++s) {
                    if (!part[s].used)
                        continue;
                    const float *const from = parts + s * kPartFloats<D, R>;
                    const float h = ex2(from[2 * r] - m);
                    const float4 x = *reinterpret_cast<const float4 *>(from + 2 * R + r * (D + 4) + 4 * c);
                    l += from[2 * r + 1] * h;
                    o.x += x.x * h, o.y += x.y * h, o.z += x.z * h, o.w += x.w * h;
                }
                if (whole) {
                    const float by = 1.f / l;
                    uint2 y = make_uint2(narrow<T>(within<T>(o.x * by), within<T>(o.y * by)),
                                         narrow<T>(within<T>(o.z * by), within<T>(o.w * by)));
                    *reinterpret_cast<uint2 *>(static_cast<T *>(p.o) + rows.b * p.o_stride +
                                               (int64_t)(rows.head + r) * D + 4 * c) = y;
                    if (c == 0 && p.lse != nullptr)
                        p.lse[(int64_t)rows.b * p.n_heads + rows.head + r] = 0.6931471805599453f * (m + log2f(l));
                } else {
                    *reinterpret_cast<float4 *>(left + 2 * R + r * (D + 4) + 4 * c) = o;
                    if (c == 0) {
                        left[2 * r] = m;
                        left[2 * r + 1] = l;
                    }
                }
            }
            s0 = s1;
        }
        if (!p.unsplit)
            return;
        __syncthreads();
    }
}

// The parts that several blocks left of an item: a block for each item and kJoinWarps / per_row rows, per_row warps to
// a row, a lane for D / 32 columns.
constexpr int kJoinWarps = 8;

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kJoinWarps * 32)
kv8_join_kernel(const __grid_constant__ AttnParams p, int per_row)
{
    constexpr int R = 8 * NT, E = D / 32, kAhead = 8;
    __shared__ Lengths all;
    __shared__ float got[kJoinWarps][D + 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Shape shape(p, R);
    // the lengths may be read before the wait: the kernel in front, which has waited itself, only
    // reads them
    read_lengths(all, p.kv_len, p.batch, p.max_kv, nullptr,
                 [&](int len) { return Shape::units(len) * shape.per_request; });
    const int b = blockIdx.x / shape.per_request, item = blockIdx.x - b * shape.per_request;
    const int units = all.before[p.batch], own = Shape::units(all.len[b]);
    const int u = all.before[b] + item * own;
    const int c0 = all.len[b] < 0 ? 0 : attn::cta_of(units, p.ctas, u);
    const int c1 = all.len[b] < 0 ? 0 : attn::cta_of(units, p.ctas, u + own - 1);
    pdl_wait_and_release();
    if (c0 == c1)
        return;
    const Rows<R> rows(p, shape, b, item);
    const int some = kJoinWarps / per_row, r = blockIdx.y * some + warp / per_row, first = warp % per_row;
    const bool on = r < rows.n;
    float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
        o[e] = 0.f;
    // up to 32 parts at a time: a lane reads one's m and l, all lanes its columns
    for (int i0 = first; on && i0 < c1 - c0 + 1; i0 += 32 * per_row) {
        const int c = c0 + i0 + lane * per_row;
        const bool here = c <= c1 && attn::has_units(units, p.ctas, c);
        const float *const from = p.part + (int64_t)(c == c0 ? 2 * c + 1 : 2 * c) * kPartFloats<D, R>;
        float pm = -INFINITY, pl = 0.f;
        if (here) {
            pm = from[2 * r];
            pl = from[2 * r + 1];
        }
        const unsigned there = __ballot_sync(0xffffffffu, here);
        float top = pm;
#pragma unroll
        for (int x = 16; x > 0; x >>= 1)
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        top = fmaxf(top, m);
        const float h = here ? ex2(pm - top) : 0.f, h0 = m == -INFINITY ? 0.f : ex2(m - top);
        float sum = pl * h;
#pragma unroll
        for (int x = 16; x > 0; x >>= 1)
            sum += __shfl_xor_sync(0xffffffffu, sum, x);
        l = l * h0 + sum;
        m = top;
#pragma unroll
        for (int e = 0; e < E; ++e)
            o[e] *= h0;
        const int count = 32 - __clz(there);
        for (int j0 = 0; j0 < count; j0 += kAhead) {
            float x[kAhead][E];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const uint64_t at = __shfl_sync(0xffffffffu, (unsigned long long)from, (j0 + j) & 31);
                const float *const y = reinterpret_cast<const float *>(at) + 2 * R + r * (D + 4) + lane * E;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    x[j][e] = (there >> ((j0 + j) & 31)) & 1 ? y[e] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const float hj = __shfl_sync(0xffffffffu, h, (j0 + j) & 31);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    o[e] = fmaf(x[j][e], hj, o[e]);
            }
        }
    }
    if (per_row > 1) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            got[warp][lane * E + e] = o[e];
        if (lane == 0) {
            got[warp][D] = m;
            got[warp][D + 1] = l;
        }
        __syncthreads();
        if (first != 0)
            return;
        for (int x = 1; x < per_row; ++x)
            m = fmaxf(m, got[warp + x][D]);
        l = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e)
            o[e] = 0.f;
        for (int x = 0; x < per_row; ++x) {
            if (got[warp + x][D] == -INFINITY)
                continue;
            const float h = ex2(got[warp + x][D] - m);
            l += got[warp + x][D + 1] * h;
#pragma unroll
            for (int e = 0; e < E; ++e)
                o[e] = fmaf(got[warp + x][lane * E + e], h, o[e]);
        }
    }
    if (!on)
        return;
    const float by = 1.f / l;
    T *const to = static_cast<T *>(p.o) + rows.b * p.o_stride + (int64_t)(rows.head + r) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2)
        reinterpret_cast<uint32_t *>(to)[e / 2] = narrow<T>(within<T>(o[e] * by), within<T>(o[e + 1] * by));
    if (lane == 0 && p.lse != nullptr)
        p.lse[(int64_t)rows.b * p.n_heads + rows.head + r] = 0.6931471805599453f * (m + log2f(l));
}

template <typename T, int D, int NT>
cudaError_t launch(const AttnParams &p, const Kv8Cache &cache, cudaStream_t s)
{
    static std::atomic<uint64_t> done{0};
    const size_t smem = 2 * kWarps * kPartFloats<D, 8 * NT> * sizeof(float);
    cudaError_t e = launch_pdl_big_smem(kv8_decode_kernel<T, D, NT>, dim3((unsigned)p.ctas), dim3(kThreads), smem, s,
                                        done, p, cache);
    if (e != cudaSuccess || !p.joined)
        return e;
    int per_row = 1;
    while (per_row < kJoinWarps && per_row * 8 < p.parts)
        per_row *= 2;
    const int rows = p.group < 8 * NT ? p.group : 8 * NT;
    const dim3 grid((unsigned)(p.batch * Shape(p, 8 * NT).per_request), (unsigned)((rows * per_row + kJoinWarps - 1) / kJoinWarps));
    return launch_pdl(kv8_join_kernel<T, D, NT>, grid, dim3(kJoinWarps * 32), 0, s, p, per_row);
}

template <typename T>
cudaError_t launch(const AttnParams &p, const Kv8Cache &cache, int d, cudaStream_t s)
{
    if (p.group > 8)
        return d == 128 ? launch<T, 128, 2>(p, cache, s) : launch<T, 64, 2>(p, cache, s);
    return d == 128 ? launch<T, 128, 1>(p, cache, s) : launch<T, 64, 1>(p, cache, s);
}

}  // namespace
}  // namespace kv8

int64_t plan_kv8_decode(AttnParams &p, int d, int sm_count)
{
    using namespace kv8;
    const int rows = p.group > 8 ? 16 : 8;
    const Shape shape(p, rows);
    const int64_t items = (int64_t)p.batch * shape.per_request, longest = Shape::units(p.max_kv);
    if (items * longest > INT_MAX)
        return -1;
    int most = sm_count * (rows == 8 ? 2 : 1);
    if (most > kAttnMaxCtas)
        most = kAttnMaxCtas;
    // a tile to a warp
    int64_t ctas = (items * longest + kWarps - 1) / kWarps;
    ctas = ctas < most ? ctas : most;
    if (longest <= 4 * kWarps)
        p.unsplit = 1;
    p.joined = !p.unsplit;
    if (p.unsplit)
        ctas = items < most ? items : most;
    p.ctas = (int)ctas;
    p.parts = (int)(longest / (items * longest / ctas > 0 ? items * longest / ctas : 1)) + 2;
    const int64_t part = sizeof(float) * (2 * rows + rows * (d + 4));
    return p.joined ? 2 * ctas * part : 0;
}

cudaError_t launch_kv8_decode(const AttnParams &p, const Kv8Cache &cache, int d, int dtype, cudaStream_t s)
{
    return dtype == HS_FP16 ? kv8::launch<__half>(p, cache, d, s) : kv8::launch<__nv_bfloat16>(p, cache, d, s);
}

}  // namespace hs
