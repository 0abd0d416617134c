// One decode step over the 8-bit cache (the FP8 KV setting, Table 1 of the paper).
//
// Per query row, with s_j = scale log2(e) q . k_j:  m a number near max s_j, l = sum 2^(s_j - m),
// a = sum 2^(s_j - m) v_j in float32; o = a / l, lse = ln 2 (m + log2 l).  m follows the maximum when a tile
// exceeds it by more than 2^8.
//
// Bytes to numbers.  E4M3 lies within binary16, so keys and values become binary16 without loss on their way
// from the load to the tensor core.  A key's scale is a factor of its scores; a value's one goes into its
// weight, w_j = 2^(s_j - m) 2^(7 - E) scale_j with 2^E the largest scale so far, so that weights are at most 2^15 and one is
// rounded to nothing only below 2^-32 of the largest (a weight is the sum of two such numbers).  A bf16 q is scaled to binary16 by a power of two
// for each row.
//
// Shares.  A tile is a group of 16 tokens.  Every warp has a contiguous run of tiles of its own, shared out
// evenly over all warps of the GPU from the device lengths, with no hand-over until its end.  A warp's lane requests its
// next tiles by TMA (they land in swizzled rows, so that the operands are read without bank conflicts, in whatever order
// of d and tokens suits that); per tile S^T = K Q^T (16 tokens x 8 rows to an instruction), the weights' matrix is
// turned between lanes, O^T += V^T W^T.  The warps of a block join their parts of an
// item (request, KV head, 8 or 16 query rows), and an item with tiles in several blocks leaves a part
// for each in the workspace, which a second kernel joins.  With `unsplit`, and where the bound is short,
// a block takes whole items instead.
//
// Few rows share a tile's bytes (the heads of one KV head), so the step is bound by HBM; products of M = 128 rows as in
// the 16-bit attention would leave most of the tensor core's rows empty, and the bytes would have to
// become numbers on a way through shared memory.  Four requests of 98k to 131k keys (943 MB) take 145 us, 6.5 TB/s, where
// the 16-bit step takes 269 to 279; 64 of 4,096 keys of 8 heads 90 us, 5.9 TB/s; 32 ragged ones 34 us, of which HBM
// accounts for 22 (3.5 us until the first tiles are there, 2 to 5 for the ends and the join's launch, 2 for the join); one
// of 4,600 keys 8.9 us, latency.  16 rows to a KV head (169 us for 799 MB, 4.7 TB/s) and heads of 64 (59 us for 268 MB) are
// bound by instructions: 475 and 320 a tile and warp (395 for 8 rows of 128), 64 and 32 of them conversions of keys
// and values, with 2 to 4 warps to a scheduler.
//
// What was tried, against the ring when it was new: loads into registers (two blocks of 8 warps to an SM: 5 % more for the long
// ones, 15 for heads of 64, 30 for 16 rows; no room for more than one tile ahead); the ring by asynchronous copies of 16
// bytes (40 %: they and the reads share one queue); prefetches into L2 (1 to 4 tiles ahead: no gain); two tiles to a step
// (1 %, but 25 for one request: code that runs once waits for its instructions).
#include "attn_ptx.cuh"
#include "kv8_walk.cuh"
#include "tensor_map.cuh"

namespace hs {
namespace kv8 {
namespace {

// Floats of a part: per row its D sums, then m, l and 2^E, in units of 2^(E - 7) of which the sums are (their own size may
// be beyond float32 where the average of the values is not), and one that keeps rows apart in the banks.
template <int D, int R>
constexpr int kPartFloats = R * (D + 4);

// The kernel's sizes.  A warp takes a step of kTiles tiles at a time; its steps arrive in a ring of its own in shared
// memory, kStages - 1 ahead.
template <int D, int NT>
struct Sizes {
    static constexpr int R = 8 * NT;
    static constexpr int kTiles = D == 128 && NT == 1 ? 1 : 2;
    static constexpr int kWarps = D == 128 ? (NT == 1 ? 12 : 8) : NT == 1 ? 16 : 12;
    static constexpr int kStages = D == 128 ? (NT == 1 ? 3 : 2) : NT == 1 ? 2 : 3;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kPlaneBytes = kGroup * D, kTileBytes = 2 * kPlaneBytes;
    static constexpr int kStageBytes = kTiles * kTileBytes, kRingBytes = kStages * kStageBytes;
    static_assert(kStageBytes % 1024 == 0 && kRingBytes >= (int)sizeof(float) * kPartFloats<D, R>);
    // beside the rings a part for each warp
    static constexpr size_t smem(int warps)
    {
        return (size_t)warps * (kRingBytes + sizeof(float) * kPartFloats<D, R>) + 1024;
    }
};

// one of a block's parts
struct Part {
    int32_t item;                 // request * items of a request + item; -1: none
    int16_t starts, ends;         // with the item's first and last tile
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 4 bytes to shared memory
__device__ __forceinline__ void copy4(uint32_t to, const void *from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}

__device__ __forceinline__ void commit()
{
    asm volatile("cp.async.commit_group;" ::: "memory");
}

// until all but the last N groups have arrived
template <int N>
__device__ __forceinline__ void arrived()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
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

// tiles of an item
__host__ __device__ __forceinline__ int units_of(int len)
{
    return len > 0 ? groups_of(len) : 1;          // an empty row is written by someone
}

// the rows of an item (KV head * row tiles + row tile) of request b
template <int R>
struct Rows {
    int b, head, n;               // head: of the first row
    __device__ __forceinline__ Rows(const AttnParams &p, const Kv8Plan &plan, int b_, int item) : b(b_)
    {
        const int kvh = plan.by_row_tiles.div(item), rt = item - kvh * plan.row_tiles;
        head = kvh * p.group + rt * R;
        n = min(R, p.group - rt * R);
    }
};

// A warp's part of an item: NT tiles of 8 rows.  A lane (g = lane / 4, t = lane % 4) has the tokens g and g + 8 of
// scores and the columns [g D/8, (g + 1) D/8) of sums, of the rows 2 t and 2 t + 1 of each tile.
template <typename T, int D, int NT>
struct Warp {
    static constexpr int R = 8 * NT, C = D / 64;
    // Numbers to a weight.  One binary16 would cost an fp16 output as much as its own rounding (3.1e-4 of it, 2-norm, instead
    // of 2.1e-4, which the output's alone makes), and a bf16 output whose keys' shares cancel several steps.  The second
    // product takes 2 to 3 % of the time, 4 with heads of 64, 8 with more than 8 rows.
    static constexpr int H = 2;
    uint32_t q[C * 4][NT][2];
    float factor[NT][2];          // of scores, beside the keys' scale
    float m[NT][2], l[NT][2];
    float o[D / 16][NT][4];
    float top;                    // 2^E, 2^-126 at least

    // the queries as they are
    __device__ __forceinline__ static void load(uint32_t (&x)[NT][C][8], const AttnParams &p, const Rows<R> &rows, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool on = n * 8 + g < rows.n;
            const T *const row = static_cast<const T *>(p.q) + rows.b * p.q_stride +
                                 (int64_t)(rows.head + n * 8 + g) * D + t * 16 * C;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint4 y = on ? reinterpret_cast<const uint4 *>(row + c * 16)[i] : make_uint4(0, 0, 0, 0);
                    x[n][c][4 * i] = y.x, x[n][c][4 * i + 1] = y.y, x[n][c][4 * i + 2] = y.z, x[n][c][4 * i + 3] = y.w;
                }
        }
    }

    __device__ __forceinline__ void begin(uint32_t (&raw)[NT][C][8], const AttnParams &p, int lane)
    {
        const int t = lane & 3;
        top = 0x1p-126f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            uint32_t (&x)[C][8] = raw[n];
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
                    q[c * 4 + i / 2][n][i & 1] = x[c][i];
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

    // scores of a tile: k[c][i] the 16 bytes [16 (C t + c), + 16) of tokens token_of(g + 8 i)
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

    // the scores of N tiles into weights, as the second product's operand; scale: of the tiles' values
    template <int N>
    __device__ __forceinline__ void weights(const float (&s)[N][NT][4], const float (&scale)[N], uint32_t (&w)[N][NT][H][2])
    {
        float x[NT][2];
        bool more = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[n][i] = fmaxf(s[0][n][i], s[0][n][i + 2]);
#pragma unroll
                for (int a = 1; a < N; ++a)
                    x[n][i] = fmaxf(x[n][i], fmaxf(s[a][n][i], s[a][n][i + 2]));
                more = more || x[n][i] > m[n][i] + 8.f;
            }
        float most = scale[0];
#pragma unroll
        for (int a = 1; a < N; ++a)
            most = fmaxf(most, scale[a]);
        if (__any_sync(0xffffffffu, more || most > top)) {
            float h0 = 1.f;
            if (most > top) {
                // a power of two even where the cache's scale is none
                const float up = __uint_as_float(__float_as_uint(most) & 0x7f800000u);
                h0 = top * inverse(up);
                top = up;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float y = x[n][i];
                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 4));
                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 8));
                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 16));
                    float h = 1.f;
                    // by the row's own scores, whichever row brought the warp here
                    if (y > m[n][i] + 8.f) {
                        h = ex2(m[n][i] - y);
                        m[n][i] = y;
                        l[n][i] *= h;
                    }
                    h *= h0;
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        o[d][n][i] *= h;
                        o[d][n][i + 2] *= h;
                    }
                }
        }
        const float down = inverse(top);                   // 128 times it may be beyond float32
#pragma unroll
        for (int a = 0; a < N; ++a) {
            const float by = scale[a] * down * 128.f;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[i] = ex2(s[a][n][i] - m[n][i & 1]);
                    l[n][i & 1] += y[i];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float y0 = y[2 * i] * by, y1 = y[2 * i + 1] * by;
                    const uint32_t z = narrow<__half>(y0, y1);
                    const float2 f = widen<__half>(z);
                    w[a][n][0][i] = transposed(z);
                    w[a][n][1][i] = transposed(narrow<__half>(y0 - f.x, y1 - f.y));
                }
            }
        }
    }

    // sums of a tile: v[i] the bytes [g D/8, + D/8) of the tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
    template <int N>
    __device__ __forceinline__ void sums(const uint32_t (&v)[4][N], const uint32_t (&w)[NT][H][2])
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
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    mma(o[2 * i][n], a0, a1, a2, a3, w[n][h][0], w[n][h][1]);
                    mma(o[2 * i + 1][n], b0, b1, b2, b3, w[n][h][0], w[n][h][1]);
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
                const float by = l[n][i] == 0.f ? 0.f : 0x1p-7f / l[n][i];
                uint32_t x[D / 16];
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
                    x[j] = narrow_finite<T>(sum(n, i, 2 * j) * by * top, sum(n, i, 2 * j + 1) * by * top);
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
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float *const row = part + (n * 8 + 2 * t + i) * (D + 4);
                if (g == 0)
                    *reinterpret_cast<float4 *>(row + D) = make_float4(m[n][i], l[n][i], top, 0.f);
                float4 *const to = reinterpret_cast<float4 *>(row + g * (D / 8));
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
                    to[j] = make_float4(sum(n, i, 4 * j), sum(n, i, 4 * j + 1), sum(n, i, 4 * j + 2), sum(n, i, 4 * j + 3));
            }
    }
};

// A tile's token that stands in row i of the products (tokens may go in any order): with 64 bytes to a token two of them
// share a 128-byte row of shared memory, and neighbours in it are neighbours in i.
template <int D>
__device__ __forceinline__ int token_of(int i)
{
    return D == 128 ? i : ((i & 7) >> 1) * 4 + (i >> 3) * 2 + (i & 1);
}

// The loads of a warp's run, ahead of its products.
template <int D, int NT>
struct Loader {
    using S = Sizes<D, NT>;
    const AttnParams &p;
    const Kv8Cache &cache;
    const CUtensorMap &map;
    const Lengths &all;
    const Kv8Plan &plan;
    const uint32_t ring, bars, scales;   // in shared memory
    const int lane;
    int left = 0;                 // units of the run not asked for
    int b, item, tile, len;       // the next one's item
    int stage = 0;
    int first = 0, ids = 0;       // the page of lane 0's id

    __device__ __forceinline__ void begin(int left_, int b_, int item_, int tile_, int len_)
    {
        left = left_, b = b_, item = item_, tile = tile_, len = len_;
        first = -64;
    }
    // the next step.  What lies in the ring stays where a page is none (that request's results mean nothing)
    __device__ __forceinline__ void issue()
    {
        if (left > 0) {
            const int per = units_of(len), n = min(S::kTiles, min(per - tile, left));
            const int shift = cache.page_shift - 4, head_plane = 2 * plan.by_row_tiles.div(item);
            const uint32_t bar = bars + 8 * stage, to = ring + stage * S::kStageBytes;
#pragma unroll 1
            for (int a = 0; a < S::kTiles; ++a) {
                int id = -1;
                const int page = (tile + a) >> shift, in_page = (tile + a) & ((1 << shift) - 1);
                if (a < n && len > 0) {
                    if ((unsigned)(page - first) >= 32) {
                        first = page;
                        ids = page + lane <= (len - 1) >> cache.page_shift ? __ldg(p.table + b * p.max_pages + page + lane) : 0;
                        if (ids < 0 || ids >= cache.num_blocks) {
                            report(p.d_err, HS_DEVERR_BLOCK_OOB);
                            ids = -1;
                        }
                    }
                    id = __shfl_sync(0xffffffffu, ids, page - first);
                }
                if (id >= 0 && lane < 2) {
                    float *at;
                    group_at<D>(cache, id, in_page, head_plane, &at);
                    copy4(scales + (stage * S::kTiles + a) * 8 + 4 * lane, at + (lane << shift));
                }
                if (lane == 0) {
                    ptx::mbar_arrive_expect_tx(bar, id >= 0 ? S::kTileBytes : 0);
                    if (id >= 0) {
                        const int y = id * (int)(cache.block_bytes / 128) +
                                      ((head_plane << shift) + in_page) * (S::kPlaneBytes / 128);
                        ptx::tma_load_2d(to + a * S::kTileBytes, &map, 0, y, bar);
                        ptx::tma_load_2d(to + a * S::kTileBytes + S::kPlaneBytes, &map, 0,
                                         y + (S::kPlaneBytes / 128 << shift), bar);
                    }
                }
            }
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
            left -= n;
            tile += n;
            if (tile == per && left > 0) {
                tile = 0;
                first = -64;
                if (++item == plan.items) {
                    item = 0;
                    do
                        ++b;
                    while (all.before[b + 1] == all.before[b]);
                    len = all.len[b];
                }
            }
        }
        commit();
    }
};

// the products of a step: n tiles from `tile` on, of an item with `len` tokens
template <typename T, int D, int NT>
__device__ __forceinline__ void step(Warp<T, D, NT> &w, const uint8_t *at, const float *scales, int tile, int n, int len,
                                     int lane)
{
    using S = Sizes<D, NT>;
    constexpr int C = D / 64, N = S::kTiles;
    const int g = lane >> 2, t = lane & 3;
    float s[N][NT][4], v_scale[N];
    uint32_t x[N][NT][Warp<T, D, NT>::H][2];
    // a 128-byte row's 16-byte chunk c lies at c ^ (row & 7)
    const int k_row = D == 128 ? g : g & 6, k_chunk = D == 128 ? 2 * t : (g & 1) * 4 + t;
#pragma unroll
    for (int a = 0; a < N; ++a) {
        uint4 k[C][2];
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = D == 128 ? k_row + 8 * j : k_row + j;
                k[c][j] = *reinterpret_cast<const uint4 *>(at + a * S::kTileBytes + row * 128 + (((k_chunk + c) ^ (row & 7)) << 4));
            }
        w.scores(k, scales[2 * a], s[a]);
        v_scale[a] = a < n ? scales[2 * a + 1] : 0.f;
    }
    const bool tail = n < N || len - tile * kGroup < N * kGroup;
    if (tail) {
#pragma unroll
        for (int a = 0; a < N; ++a) {
            const int left = a < n ? len - (tile + a) * kGroup : 0;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (token_of<D>(g + 8 * (c >> 1)) >= left)
                        s[a][i][c] = -INFINITY;
        }
    }
    w.template weights<N>(s, v_scale, x);
#pragma unroll
    for (int a = 0; a < N; ++a) {
        const uint8_t *const from = at + a * S::kTileBytes + S::kPlaneBytes;
        uint32_t v[4][D / 32];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (D == 128) {
                const int row = 2 * t + (j & 1) + (j >> 1) * 8;
                const uint4 y = *reinterpret_cast<const uint4 *>(from + row * 128 + ((g ^ (row & 7)) << 4));
                v[j][0] = y.x, v[j][1] = y.y, v[j][2] = y.z, v[j][3] = y.w;
            } else {
                const int row = 2 * t + (j >> 1), chunk = (j & 1) * 4 + (g >> 1);
                const uint2 y = *reinterpret_cast<const uint2 *>(from + row * 128 + ((chunk ^ row) << 4) + (g & 1) * 8);
                v[j][0] = y.x, v[j][1] = y.y;
            }
        }
        if (tail) {
            // behind the last key: values of zero (a weight of 0 times NaN is NaN)
            const int left = a < n ? len - (tile + a) * kGroup : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (token_of<D>(2 * t + (j & 1) + (j >> 1) * 8) >= left)
#pragma unroll
                    for (int c = 0; c < D / 32; ++c)
                        v[j][c] = 0;
        }
        w.sums(v, x[a]);
    }
}

// where an item's result goes that a block has the beginning but not the end of (item < 0: none), for the join
struct Split {
    int32_t item, last;                            // index of the item; the last block with a part
};

__host__ __device__ __forceinline__ int64_t parts_at(int ctas)
{
    return (int64_t)(ctas + 1) / 2 * 4;            // parts stay 16-byte aligned
}

// a row's state beside its sums, which are in units of 2^-7 unit
struct State {
    float m, l, unit;
    __device__ __forceinline__ State() : m(-INFINITY), l(0.f), unit(0x1p-126f) {}     // of no tiles
    __device__ __forceinline__ explicit State(float4 x) : m(x.x), l(x.y), unit(x.z) {}
    __device__ __forceinline__ operator float4() const { return make_float4(m, l, unit, 0.f); }
    __device__ __forceinline__ bool none() const { return m == -INFINITY && l == 0.f; }
};

// one row's result, a lane's columns c to c + 3
template <typename T, int D>
__device__ __forceinline__ void write_row(const AttnParams &p, int b, int head, int c, float4 o, const State &x)
{
    const float by = x.l == 0.f ? 0.f : 0x1p-7f / x.l;
    *reinterpret_cast<uint2 *>(static_cast<T *>(p.o) + b * p.o_stride + (int64_t)head * D + c) =
        make_uint2(narrow_finite<T>(o.x * by * x.unit, o.y * by * x.unit),
                   narrow_finite<T>(o.z * by * x.unit, o.w * by * x.unit));
    if (c == 0 && p.lse != nullptr)
        p.lse[(int64_t)b * p.n_heads + head] = 0.6931471805599453f * (x.m + log2f(x.l));
}

// Parts of a row joined by a warp: lane i has part i's state, row_of(i, i % kAhead) a lane's four columns of its sums,
// loaded kAhead at a time.
template <int kAhead, typename RowOf>
__device__ __forceinline__ float4 join(State &s, int count, RowOf row_of)
{
    float top = s.m;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1)
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
    float h = s.none() ? 0.f : ex2(s.m - top);
    s.m = top;
    s.l *= h;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1)
        s.l += __shfl_xor_sync(0xffffffffu, s.l, x);
    const float unit = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(s.unit)));
    h *= s.unit * inverse(unit);
    s.unit = unit;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int i0 = 0; i0 < count; i0 += kAhead) {
        float4 x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            x[k] = row_of(min(i0 + k, count - 1), k);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const float hi = __shfl_sync(0xffffffffu, h, (i0 + k) & 31);
            if (i0 + k < count)
                o.x = fmaf(x[k].x, hi, o.x), o.y = fmaf(x[k].y, hi, o.y), o.z = fmaf(x[k].z, hi, o.z),
                o.w = fmaf(x[k].w, hi, o.w);
        }
    }
    return o;
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(Sizes<D, NT>::kThreads, 1)
kv8_decode_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ Kv8Plan plan,
                  const __grid_constant__ Kv8Cache cache,
                  const __grid_constant__ CUtensorMap map)
{
    using S = Sizes<D, NT>;
    constexpr int R = S::R, kPart = kPartFloats<D, R>;
    extern __shared__ uint8_t shared[];
    __shared__ Lengths all;
    __shared__ Part part[2 * S::kWarps];
    __shared__ int32_t order[2 * S::kWarps], firsts[2 * S::kWarps + 1];
    __shared__ float scales[S::kWarps][S::kStages][2 * S::kTiles];
    __shared__ uint64_t bars[S::kWarps][S::kStages + 1];     // the last one is for failure-detection tests
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    uint8_t *const rings = shared + (-(intptr_t)ptx::smem_u32(shared) & 1023), *const ring = rings + warp * S::kRingBytes;
    float *const heads = reinterpret_cast<float *>(rings + warps * S::kRingBytes);
    if (lane <= S::kStages)
        ptx::mbar_init(ptx::smem_u32(&bars[warp][lane]), S::kTiles);
    ptx::fence_mbar_init();
    if (threadIdx.x == 0)
        ptx::prefetch_tensormap(&map);
    __syncwarp();
    pdl_wait_and_release();
    Loader<D, NT> loader{p, cache, map, all, plan, ptx::smem_u32(ring), ptx::smem_u32(bars[warp]),
                         ptx::smem_u32(scales[warp]), lane};
    int stage = 0, parity = 0;
    bool lost = false;                                       // a wait has run out
    if (!p.unsplit)
        read_lengths(all, p.kv_len, p.batch, p.max_kv, p.d_err,
                     [&](int len) { return units_of(len) * plan.items; });
    const Shares shares(p.unsplit ? 0 : all.before[p.batch], plan.by_ctas);

    // the block's run: its share of all units, or one whole item after the other
    for (int turn = blockIdx.x;; turn += gridDim.x) {
        int u, end, b, item, tile, len;                      // of the warp's run
        if (p.unsplit) {
            if (turn >= p.batch * plan.items)
                return;
            b = plan.by_items.div(turn);
            item = turn - b * plan.items;
            len = p.kv_len[b];
            if (len < 0 || len > p.max_kv) {
                if (threadIdx.x == 0)
                    report(p.d_err, HS_DEVERR_LENGTH);
                continue;
            }
            const int n = units_of(len);
            const Shares over(n, plan.by_warps);
            u = tile = over.begin(warp);
            end = over.begin(warp + 1);
        } else {
            u = end = b = item = tile = len = 0;
            const int u0 = shares.begin(blockIdx.x);
            const Shares over(shares.begin(blockIdx.x + 1) - u0, plan.by_warps);
            u = u0 + over.begin(warp);
            end = u0 + over.begin(warp + 1);
            if (u < end) {
                b = request_of(all, p.batch, u, lane);
                len = all.len[b];
                const int per = units_of(len);
                item = (u - all.before[b]) / per;
                tile = (u - all.before[b]) - item * per;
            }
        }
        if (lane < 2)
            part[2 * warp + lane].item = -1;
        if (u < end && !lost) {
            uint32_t raw[NT][D / 64][8];
            Warp<T, D, NT>::load(raw, p, Rows<R>(p, plan, b, item), lane);
            ptx::fence_proxy_async_smem();                   // the ring held parts
            loader.begin(end - u, b, item, tile, len);
            Warp<T, D, NT> w;
            int from = tile, n = min(units_of(len) - tile, end - u);     // the segment: tiles [from, from + n)
#pragma unroll 1
            for (int ahead = 1 - S::kStages;; ++ahead) {
                if (ahead >= 0) {
                    lost = !ptx::mbar_wait_bounded(p.stall_for_test ? loader.bars + 8 * S::kStages : loader.bars + 8 * stage,
                                                   parity, p.limit_ns);
                    arrived<S::kStages - 2>();
                    lost = __any_sync(0xffffffffu, lost);
                    __syncwarp();                            // all lanes see the scales, and have read the stage before
                    if (lost)
                        break;
                }
                loader.issue();
                if (ahead < 0)
                    continue;
                if (tile == from)
                    w.begin(raw, p, lane);
                if (len > 0)
                    step(w, ring + stage * S::kStageBytes, scales[warp][stage], tile, min(S::kTiles, from + n - tile), len, lane);
                if (++stage == S::kStages) {
                    stage = 0;
                    parity ^= 1;
                }
                tile += S::kTiles;
                if (tile < from + n)
                    continue;
                // the segment's end
                const int per = units_of(len);
                const Rows<R> rows(p, plan, b, item);
                u += n;
                w.end();
                if (n == per) {
                    w.write(p, rows, lane);
                } else {
                    // the run's last part goes over the ring, one in front of it behind the rings
                    const bool last = u == end;
                    if (last)
                        arrived<0>();
                    __syncwarp();
                    w.leave(last ? reinterpret_cast<float *>(ring) : heads + warp * kPart, lane);
                    if (lane == 0)
                        part[2 * warp + last] = Part{b * plan.items + item, from == 0, from + n == per};
                }
                if (u == end)
                    break;
                if (++item == plan.items) {
                    item = 0;
                    do
                        ++b;
                    while (all.before[b + 1] == all.before[b]);
                    len = all.len[b];
                }
                from = tile = 0;
                n = min(units_of(len), end - u);
                Warp<T, D, NT>::load(raw, p, Rows<R>(p, plan, b, item), lane);
            }
            if (lost) {
                // wait for what is on its way, and leave
                report(p.d_err, HS_DEVERR_TIMEOUT);
                while (stage != loader.stage) {
                    (void)ptx::mbar_wait_bounded(loader.bars + 8 * stage, parity, p.limit_ns);
                    if (++stage == S::kStages) {
                        stage = 0;
                        parity ^= 1;
                    }
                }
                arrived<0>();
            }
        }
        __syncthreads();

        // Join the parts of each item.  Those of an item stand one behind the other in the order of slots; every warp finds
        // the same order, and takes rows of items in turn.
        const Part mine = lane < 2 * warps ? part[lane] : Part{-1, 0, 0};
        const unsigned used = __ballot_sync(0xffffffffu, mine.item >= 0);
        if (mine.item >= 0)
            order[__popc(used & ((1u << lane) - 1))] = lane;
        __syncwarp();
        const int count = __popc(used), slot = lane < count ? order[lane] : 0;
        const int items = __shfl_sync(0xffffffffu, mine.item, slot);
        const int in_front = __shfl_up_sync(0xffffffffu, items, 1);
        const bool begins = lane < count && (lane == 0 || items != in_front);
        const unsigned begin = __ballot_sync(0xffffffffu, begins);
        if (begins)
            firsts[__popc(begin & ((1u << lane) - 1))] = lane;
        const int chains = __popc(begin);
        if (lane == 0)
            firsts[chains] = count;
        __syncwarp();
        const int live = min(R, p.group);                   // rows of an item at most
        for (int job = warp; job < chains * live; job += warps) {
            const int c = job / live, r = job - c * live, i0 = firsts[c], n = firsts[c + 1] - i0;
            const int own = order[i0 + min(lane, n - 1)];
            const float *at = own & 1 ? reinterpret_cast<const float *>(rings + (own >> 1) * S::kRingBytes)
                                      : heads + (own >> 1) * kPart;
            const Part a = part[own];
            const int it = a.item, bb = plan.by_items.div(it);
            const bool starts = __shfl_sync(0xffffffffu, a.starts, 0), ends = __shfl_sync(0xffffffffu, a.ends, n - 1);
            const Rows<R> rows(p, plan, bb, it - bb * plan.items);
            if (r >= rows.n || (!(starts && ends) && !p.joined))       // the latter: a wait has run out
                continue;
            at += r * (D + 4);
            State s;
            if (lane < n)
                s = State(*reinterpret_cast<const float4 *>(at + D));
            const int col = lane * 4 % D;                   // 64 columns: the second half of the lanes repeats the first
            const float4 o = join<4>(s, n, [&](int i, int) {
                const int from = __shfl_sync(0xffffffffu, (int)(at - heads), i);
                return *reinterpret_cast<const float4 *>(heads + from + col);
            });
            if (lane * 4 >= D)
                continue;
            if (starts && ends) {
                write_row<T, D>(p, bb, rows.head + r, col, o, s);
                continue;
            }
            float *const to = p.part + parts_at(gridDim.x) + (int64_t)(2 * blockIdx.x + starts) * kPart + r * (D + 4);
            *reinterpret_cast<float4 *>(to + col) = o;
            if (lane == 0)
                *reinterpret_cast<float4 *>(to + D) = s;
        }
        if (!p.unsplit) {
            if (threadIdx.x == 0) {
                // the item that goes on in the next block
                Split x{-1, 0};
                if (chains > 0) {
                    const Part a = part[order[firsts[chains - 1]]], z = part[order[count - 1]];
                    if (a.starts && !z.ends) {
                        const int bb = plan.by_items.div(a.item), per = units_of(all.len[bb]);
                        const int last = all.before[bb] + (a.item - bb * plan.items + 1) * per - 1;
                        x.item = a.item;
                        x.last = shares.of(last);
                    }
                }
                reinterpret_cast<Split *>(p.part)[blockIdx.x] = x;
            }
            return;
        }
        __syncthreads();
    }
}

// The parts that several blocks left of an item: the block x in which the item begins, kJoinWarps / per_row rows, per_row
// warps to a row.
constexpr int kJoinWarps = 8;

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kJoinWarps * 32)
kv8_join_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ Kv8Plan plan)
{
    constexpr int R = 8 * NT, kPart = kPartFloats<D, R>, kAhead = 4;
    __shared__ float4 sums[kJoinWarps][32];
    __shared__ float4 states[kJoinWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per_row = plan.per_row;
    const int r = blockIdx.y * (kJoinWarps / per_row) + warp / per_row, first = warp % per_row;
    const int col = lane * 4 % D;
    pdl_wait_and_release();
    const Split x = reinterpret_cast<const Split *>(p.part)[blockIdx.x];
    if (x.item < 0)
        return;
    const int b = plan.by_items.div(x.item);
    const Rows<R> rows(p, plan, b, x.item - b * plan.items);
    State s;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    // up to 32 parts at a time, the sums of the first ones on their way with the states
    for (int c0 = blockIdx.x + first; r < rows.n && c0 <= x.last; c0 += 32 * per_row) {
        auto at = [&](int i) {
            const int c = c0 + i * per_row;
            return p.part + parts_at(plan.ctas) + (int64_t)(c == (int)blockIdx.x ? 2 * c + 1 : 2 * c) * kPart + r * (D + 4);
        };
        auto row = [&](int i) { return *reinterpret_cast<const float4 *>(at(i) + col); };
        const int count = min(32, (x.last - c0) / per_row + 1);
        float4 ahead[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            ahead[i] = row(min(i, count - 1));
        State part;
        if (lane < count)
            part = State(*reinterpret_cast<const float4 *>(at(lane) + D));
        const float4 y = join<kAhead>(part, count, [&](int i, int k) { return i < kAhead ? ahead[k] : row(i); });
        const float top = fmaxf(s.m, part.m), unit = fmaxf(s.unit, part.unit);
        float h = s.none() ? 0.f : ex2(s.m - top), hy = part.none() ? 0.f : ex2(part.m - top);
        s.l = s.l * h + part.l * hy;
        h *= s.unit * inverse(unit);
        hy *= part.unit * inverse(unit);
        o.x = o.x * h + y.x * hy, o.y = o.y * h + y.y * hy, o.z = o.z * h + y.z * hy, o.w = o.w * h + y.w * hy;
        s.m = top;
        s.unit = unit;
    }
    if (per_row > 1) {
        sums[warp][lane] = o;
        if (lane == 0)
            states[warp] = s;
        __syncthreads();
        if (first != 0)
            return;
        s = lane < per_row ? State(states[warp + lane]) : State();
        o = join<2>(s, per_row, [&](int i, int) { return sums[warp + i][lane]; });
    }
    if (r < rows.n && lane * 4 < D)
        write_row<T, D>(p, b, rows.head + r, col, o, s);
}

// The cache as rows of 128 bytes: a copy takes a group of one head's plane, which lands in swizzled rows (16-byte chunk c
// of row r at c ^ (r & 7)), so that a warp reads the products' operands without bank conflicts.
template <int D>
bool encode(CUtensorMap *m, const Kv8Cache &cache)
{
    auto fn = attn::encode_fn();
    if (fn == nullptr)
        return false;
    cuuint64_t dim[2] = {128, (cuuint64_t)(cache.num_blocks * (cache.block_bytes / 128))};
    cuuint64_t stride[1] = {128};
    cuuint32_t box[2] = {128, kGroup * D / 128}, one[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, cache.base, dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, int NT>
cudaError_t launch(const AttnParams &p, const Kv8Plan &plan, const Kv8Cache &cache, cudaStream_t s)
{
    using S = Sizes<D, NT>;
    static std::atomic<uint64_t> done{0};
    CUtensorMap map;
    if (!encode<D>(&map, cache))
        return cudaErrorInvalidValue;
    const cudaError_t e = launch_pdl_smem_limit(kv8_decode_kernel<T, D, NT>, dim3((unsigned)plan.ctas),
                                                dim3((unsigned)plan.warps * 32), S::smem(plan.warps), S::smem(S::kWarps),
                                                s, done, p, plan, cache, map);
    if (e != cudaSuccess || !p.joined)
        return e;
    const int rows = p.group < S::R ? p.group : S::R;
    return launch_pdl(kv8_join_kernel<T, D, NT>,
                      dim3((unsigned)plan.ctas, (unsigned)((rows * plan.per_row + kJoinWarps - 1) / kJoinWarps)),
                      dim3(kJoinWarps * 32), 0, s, p, plan);
}

template <typename T>
cudaError_t launch(const AttnParams &p, const Kv8Plan &plan, const Kv8Cache &cache, int d, cudaStream_t s)
{
    if (p.group > 8)
        return d == 128 ? launch<T, 128, 2>(p, plan, cache, s) : launch<T, 64, 2>(p, plan, cache, s);
    return d == 128 ? launch<T, 128, 1>(p, plan, cache, s) : launch<T, 64, 1>(p, plan, cache, s);
}

template <int D, int NT>
int64_t make_plan(AttnParams &p, Kv8Plan &plan, int sm_count)
{
    using S = Sizes<D, NT>;
    plan.row_tiles = (p.group + S::R - 1) / S::R;
    plan.items = plan.row_tiles * p.n_kv;
    const int64_t items = (int64_t)p.batch * plan.items, longest = units_of(p.max_kv);
    if (items * longest > INT_MAX)
        return -1;
    // Whole items: as many warps to each as the SMs have for it, and as it has steps.  They save the join and the walk over
    // lengths, 2 to 5 us, and cost what the longest item takes its warps above an even share.  128 short requests of 2 heads
    // 7.1 us instead of 12.9 split, 300 of 8 heads of up to 150 keys 23.9 instead of 29.7, 32 of 4 heads of up to 2,000 keys
    // as fast either way (16.5); but with one warp to an item 128 of 8 heads of up to 400 keys (25 tiles) 29.4 instead of 24.3,
    // and where half of the SMs would have none, one request of 4 heads of 1,500 keys (8 tiles to a warp) 12.3 instead of 8.8.
    const int64_t rounds = (items + sm_count - 1) / sm_count, steps = (longest + S::kTiles - 1) / S::kTiles;
    int64_t warps = rounds < S::kWarps ? S::kWarps / rounds : 1;
    if (warps > steps)
        warps = steps;
    if (p.unsplit)
        warps = S::kWarps;
    else if (longest <= (items * 2 >= sm_count ? 12 : 4) * warps)
        p.unsplit = 1;
    p.joined = !p.unsplit;
    if (p.unsplit) {
        const int64_t most = sm_count * (S::kWarps / warps);
        plan.ctas = (int)(items < most ? items : most);
    } else {
        // A block to each SM, fewer where they would not be full: a step to a warp.  One request of one KV head and 8,000 keys
        // of 64 9.1 us in 16 blocks of 16 warps, 10.2 in 152 of two, whose many parts are joined.
        const int64_t all = (items * steps + S::kWarps - 1) / S::kWarps;
        plan.ctas = (int)(all < sm_count ? all : sm_count);
        warps = S::kWarps;
    }
    plan.warps = (int)warps;
    // about two parts to a warp of the join
    const int64_t parts = longest / (items * longest / plan.ctas > 0 ? items * longest / plan.ctas : 1) + 1;
    plan.per_row = 1;
    while (plan.per_row < kJoinWarps && plan.per_row * 2 < parts)
        plan.per_row *= 2;
    plan.by_row_tiles.set(plan.row_tiles);
    plan.by_items.set(plan.items);
    plan.by_warps.set(plan.warps);
    plan.by_ctas.set(plan.ctas);
    // two parts of a block
    return p.unsplit ? 0 : (int64_t)sizeof(float) * (parts_at(plan.ctas) + (int64_t)2 * plan.ctas * kPartFloats<D, S::R>);
}

}  // namespace
}  // namespace kv8

int64_t plan_kv8_decode(AttnParams &p, Kv8Plan &plan, int d, int sm_count)
{
    p.limit_ns = 1000000000ull;
    if (p.group > 8)
        return d == 128 ? kv8::make_plan<128, 2>(p, plan, sm_count) : kv8::make_plan<64, 2>(p, plan, sm_count);
    return d == 128 ? kv8::make_plan<128, 1>(p, plan, sm_count) : kv8::make_plan<64, 1>(p, plan, sm_count);
}

cudaError_t launch_kv8_decode(const AttnParams &p, const Kv8Plan &plan, const Kv8Cache &cache, int d, int dtype,
                              cudaStream_t s)
{
    return dtype == HS_FP16 ? kv8::launch<__half>(p, plan, cache, d, s) : kv8::launch<__nv_bfloat16>(p, plan, cache, d, s);
}

}  // namespace hs
