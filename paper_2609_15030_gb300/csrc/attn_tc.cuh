// Softmax attention over the paged cache (the full-attention layers) on tcgen05 tensor cores.
//
// Rows.  The query heads of one KV head are stacked: row r of an item is token r / group, head
// r % group, so that one tile of keys serves all of them.  An item is NG tiles of 128 rows of one
// (request, KV head); its keys are walked in tiles of 128.  The units of work are (item, key tile).
//
// Mathematics, per row, with s_j = scale * log2(e) * q . k_j:  m is a number near max s_j,
// l = sum 2^(s_j - m), a = sum 2^(s_j - m) v_j, all float32;  o = a / l, lse = ln 2 (m + log2 l).
// m follows the maximum lazily: only when a tile's maximum exceeds it by more than 8 (fp16: 15) are l
// and a rescaled by 2^(m_old - m_new), and nothing is lost, since the scale of 16-bit weights is free.  In
// fp16 m is then set 8 below the maximum: weights lie between 2^15 and 2^-24, so that a key's is rounded
// to nothing only below 2^-33 of the largest (with m at the maximum, many keys of 2^-25 each were lost).
// Weights are rounded to the element type for the product with v (the tensor core takes 16-bit
// operands); l sums them before that rounding.
// 2^(s_j - m) is one fused multiplication and addition of q . k_j, m a rounded product.  What that rounding
// takes off is the same factor of all weights of the row and cancels in o; but with m beyond 2^31 it is
// 2^+-128 and more (NaN, or weights of nothing but 0), and beyond 2^24 fp16 weights overflow.  So from 2^28 (fp16:
// 2^23) on all products are rounded before m is taken off, and the largest gets a weight of 2^0 (2^8).
//
// Schedule.  The units of all items in order are shared out evenly over the CTAs, each a
// contiguous run, so that one long request or many ragged ones fill the SMs alike.  An item whose
// keys fall to several CTAs leaves (m, l, a) of each in the workspace and a second kernel joins
// them.  With `unsplit` a CTA takes the whole items that begin in its run.
//
// Warps.  Per tile of rows one group of four softmax warps (thread = row = TMEM lane) and a warp that
// issues its MMAs; one warp that loads keys and values by TMA; the others look after values at
// masked places.  Per key tile and group: S = Q K^T into TMEM; the group reads it, writes the
// weights over it as 16-bit pairs; O += P V with P as the TMEM operand.  With
// two groups the tensor core works on one while the other is in its softmax.
//
// Values at masked places.  A weight of zero times a NaN or an infinity is NaN, so v must be finite
// wherever some row of the tile does not attend: rows behind the last key are zeroed in shared
// memory, and keys that only some rows see (the causal diagonal) are searched; a value there that
// is not finite is zeroed and noted, and the rows that do see it get NaN in its column at the end.
//
// What bounds it.  A key tile's two products take a group 533 ns of tensor core (M = N = 128, 8,192
// operations a clock, 1.92 GHz), its softmax 650 ns (128 exponentials a thread at 8 lanes a clock
// and scheduler take 270; the rest are maxima, sums, conversions and the passage through TMEM), and
// some 250 ns go into the hand-overs, so a pair of tiles takes 1.45 us where the tensor core alone
// would take 1.07; with a shorter softmax (two threads to a row) registers spilled and it took 2.3.
// Two 16k-token prompts of 32 heads: 2.7 to 3.06 ms, 1,640 to 1,440 TFLOP/s, at the power limit (a cuBLAS
// product sustains 1,692 there); two of 8k tokens 676 us, 1,626.  Heads of 64 have half the products to the
// same softmax: 1.2 us a pair of tiles, 1,040 TFLOP/s.  A decode step is bound by HBM where its contexts are long
// (four requests at 98k to 131k keys: 269 to 275 us, 7.0 to 6.85 TB/s), a short call by latency: 3.5 us until the first
// scores, 0.7 us of softmax, 1.3 us for sums of 256 rows that go to the workspace, 3 to 4 us for the join.
// A segment costs what two tiles cost beside its own: its description, queries, and outputs, code that runs
// once and waits for its instructions.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_ptx.cuh"
#include "attn_walk.cuh"
#include "tensor_map.cuh"

namespace hs {
namespace attn {

using namespace ptx;

constexpr float kLn2 = 0.6931471805599453f;
constexpr uint64_t kTimeoutNs = 1000000000ull;       // for copies and MMAs in flight to end

// ---- shapes of a launch --------------------------------------------------------------------

template <int D, int NG>
struct Cfg {
    static constexpr int kTile = kKeys * D * 2;            // bytes of a tile of keys, values or rows
    // two groups: one CTA per SM, as many stages as fit; one group: two CTAs per SM
    static constexpr int kStages = NG == 2 ? (D == 128 ? 5 : 8) : (D == 128 ? 2 : 5);
    static constexpr int kSoftmax = NG * 4;               // warps
    static constexpr int kThreads = (kSoftmax + 4) * 32;
    // registers of a softmax thread and of another one, out of those of the launch (65,536 over the
    // resident threads, a multiple of 8): 256 x 216 + 128 x 72 = 384 x 168 and
    // 128 x 200 + 128 x 56 = 256 x 128
    static constexpr int kRegs = NG == 2 ? 168 : 128;
    static constexpr int kMoreRegs = NG == 2 ? 216 : 200, kLessRegs = NG == 2 ? 72 : 56;
    static_assert(kSoftmax * 32 * kMoreRegs + 128 * kLessRegs <= kThreads * kRegs, "");
    // of each group S in 128 columns, O in D, and with D = 64 the weights in 64 of their own, so that the
    // next scores need not wait for the product that reads these
    static constexpr int kTmemCols = NG == 2 ? 512 : 256;
    static constexpr bool kOwnWeights = D == 64;
    static constexpr int kWeightsAt = kOwnWeights ? 192 : 0;
};

constexpr int kRing = 4;                 // segments described ahead

// One segment as the loading warp describes it to the others.  (Each of them walking by itself cost
// a softmax warp 1 to 2 us a segment, in integer divisions and cold constants.)
struct Info {
    int32_t kt0, most;                   // first key tile; tiles of the group with the most, -1: the end
    int32_t all, common;                 // keys that the last row, that every row attends to
    int32_t head0;                       // first head of the KV head
    int32_t slot_rows;                   // rows of the slot for partial results
    int64_t slot;                        // its place in the workspace (floats); -1: results are written
    struct {
        int32_t row0, key0;              // token row and keys of the group's first row's token
        int32_t head, rows;              // that row's head in the group; rows, at most 128
        int32_t keys, tiles;             // keys of its last row; its tiles in the segment
        int32_t at, unused;              // its first row in the slot
    } g[2];
};

// shared memory behind the tiles
template <int D, int NG>
struct Smem {
    uint64_t full[8], empty[8];          // a stage may be read / its MMAs are done
    uint64_t raw[8];                     // a value tile with masked places has landed
    uint64_t q_full[2], s_full[2], p_full[2], o_full[2];
    uint64_t s_read[2];                  // weights in columns of their own: the scores are in registers
    uint64_t info_full[kRing], info_empty[kRing];
    uint64_t turn[2];                    // which group's products are next
    uint64_t drain[2];
    uint32_t tmem;
    int32_t abort;
    Info info[kRing];
    union {
        int32_t len[HS_MAX_BATCH];       // decode: keys, or -1 for a length out of bounds
        struct {                         // prefill: values that are not finite, by segment
            int32_t any[kRing];
            int32_t from[kRing][D];      // first such position in the column
        } marks;
    };
};

template <int D, int NG>
constexpr int smem_bytes()
{
    return Cfg<D, NG>::kTile * (NG + Cfg<D, NG>::kStages) + (int)sizeof(Smem<D, NG>);
}
static_assert(smem_bytes<128, 2>() <= 227 * 1024 && smem_bytes<64, 2>() <= 227 * 1024, "");
static_assert(2 * (smem_bytes<128, 1>() + 1024) <= 228 * 1024 &&
              2 * (smem_bytes<64, 1>() + 1024) <= 228 * 1024, "two CTAs per SM");

// ---- element types -------------------------------------------------------------------------

template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
    static constexpr uint32_t kExp = 0x7F807F80u, kOne = 0x00800080u;
    static constexpr float kMost = 8.f, kBelow = 0.f;       // log2 of the largest weight, of a new m's
    static constexpr float kFar = 268435456.f;              // 2^28: from here on scores are rounded before m
                                                            // is taken off (a half step of 16 adds to kMost)
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    // an output in its range: what the sums give (below 2^128)
    static __device__ __forceinline__ float in_range(float x) { return x; }
    static constexpr uint32_t idesc(int N, int mn) { return idesc_bf16(128, N, mn); }
    static __device__ __forceinline__ uint32_t plus_zero_times(uint32_t z, uint32_t x)
    {
        asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(z) : "r"(x), "r"(0));
        return z;
    }
};
template <>
struct Elem<__half> {
    static constexpr uint32_t kExp = 0x7C007C00u, kOne = 0x04000400u;
    static constexpr float kMost = 15.f, kBelow = 8.f;
    static constexpr float kFar = 8388608.f;                // 2^23: two half steps of 1/4 below, and 2^15.5 fits
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    // averages of finite values are at most 65504; by the weights' rounding they come out up to 2^-11 above,
    // which would round to infinity
    static __device__ __forceinline__ float in_range(float x)
    {
        return fabsf(x) < INFINITY ? fminf(fmaxf(x, -65504.f), 65504.f) : x;
    }
    static constexpr uint32_t idesc(int N, int mn) { return idesc_f16(128, N, mn); }
    static __device__ __forceinline__ uint32_t plus_zero_times(uint32_t z, uint32_t x)
    {
        asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(z) : "r"(x), "r"(0));
        return z;
    }
};

// sign bits of the 16-bit halves whose exponent is all ones (infinities and NaN)
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x)
{
    return ((x & Elem<T>::kExp) + Elem<T>::kOne) & 0x80008000u;
}

// exchanges x of the lane with the bit `by` in its number set and y of the other
__device__ __forceinline__ void swap_chunks(uint4 &x, uint4 &y, bool upper, int by)
{
    const uint4 give = upper ? x : y;
    uint4 take;
    take.x = __shfl_xor_sync(0xffffffffu, give.x, by);
    take.y = __shfl_xor_sync(0xffffffffu, give.y, by);
    take.z = __shfl_xor_sync(0xffffffffu, give.z, by);
    take.w = __shfl_xor_sync(0xffffffffu, give.w, by);
    if (upper)
        x = take;
    else
        y = take;
}

__device__ __forceinline__ float max3(float x, float y, float z)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// ---- the kernel ----------------------------------------------------------------------------

template <typename T, int D, int NG, class Plan>
__global__ void __launch_bounds__(Cfg<D, NG>::kThreads, NG == 2 ? 1 : 2)
attn_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ Plan plan,
            const __grid_constant__ CUtensorMap map)
{
    using C = Cfg<D, NG>;
    using Sm = Smem<D, NG>;
    constexpr int kSt = C::kStages;
    constexpr int kHalf = D / 64;                    // 64-element blocks of a row
    extern __shared__ __align__(1024) uint8_t smem_raw[];   // the 128-byte swizzle's period
    const uint32_t q_at = smem_u32(smem_raw), st_at = q_at + NG * C::kTile;
    Sm &sm = *reinterpret_cast<Sm *>(smem_raw + (NG + kSt) * C::kTile);
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
    const int cta = blockIdx.x;

    auto full = [&](int i) { return smem_u32(&sm.full[i]); };
    auto empty = [&](int i) { return smem_u32(&sm.empty[i]); };
    // a bounded wait of a whole warp: false once this or another one of the CTA has run out
    volatile int32_t *const abort = &sm.abort;
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        bool ok = mbar_try_wait(bar, parity);
        if (!ok) {
            const uint64_t t0 = globaltimer_ns();
            while (!(ok = mbar_try_wait(bar, parity)) && *abort == 0) {
                if (globaltimer_ns() - t0 > p.limit_ns)
                    *abort = 1;
            }
        }
        return __all_sync(0xffffffffu, ok);
    };

    if (tid == 0) {
        for (int i = 0; i < kSt; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), NG);
            mbar_init(smem_u32(&sm.raw[i]), 1);
        }
        for (int g = 0; g < 2; ++g) {
            mbar_init(smem_u32(&sm.q_full[g]), 128);
            mbar_init(smem_u32(&sm.s_full[g]), 1);
            mbar_init(smem_u32(&sm.p_full[g]), 128);
            mbar_init(smem_u32(&sm.o_full[g]), 1);
            mbar_init(smem_u32(&sm.s_read[g]), 128);
            mbar_init(smem_u32(&sm.drain[g]), 1);
            mbar_init(smem_u32(&sm.turn[g]), 1);
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(smem_u32(&sm.info_full[i]), 1);
            mbar_init(smem_u32(&sm.info_empty[i]), C::kSoftmax + 3);
        }
        fence_mbar_init();
        sm.abort = 0;
    }
    if (warp == C::kSoftmax + 3 && lane == 0)
        prefetch_tensormap(&map);
    if (warp == C::kSoftmax)
        tmem_alloc(smem_u32(&sm.tmem), C::kTmemCols);
    pdl_wait();
    // a decode step's join takes its place as CTAs end (one step 10.2 us instead of 10.6); a prefill's does
    // not (packed drafts 13.9 us instead of 15.4)
    if (Plan::kDecode && p.joined)
        pdl_release();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t *)&sm.tmem;
    // segment k as described, and the end of this warp's use of it
    auto described = [&](uint32_t k) -> bool {
        return wait(smem_u32(&sm.info_full[k % kRing]), (k / kRing) & 1);
    };
    auto done_with = [&](uint32_t k) {
        __syncwarp();
        if (lane == 0)
            mbar_arrive(smem_u32(&sm.info_empty[k % kRing]));
    };

    // A warpgroup's four warps move their registers by one instruction, whatever each of them does then (and
    // the roles lie within the branches: behind a join of these the compiler gives all the smaller share).
    if (warp >= C::kSoftmax) {
        fewer_registers<C::kLessRegs>();
        if (warp == C::kSoftmax + 3) {
            // ---- the walk, and loads: key and value tiles in turn through the stages
            Start start;
            if constexpr (Plan::kDecode) {
                int before = 0;
                const int own = read_lengths(p, sm.len, lane, cta == 0, 0, &before);
                start = find_start<NG>(p, sm.len, own, cta, lane);
            } else {
                start = find_start<NG>(p, plan, cta);
            }
            Walk<NG, Plan> walk(p, plan, sm.len, start);
            Segment s;
            const int per = p.page_shift >= 7 ? 1 : kKeys >> p.page_shift;      // pages of a tile
            const int box = p.page_shift >= 7 ? kKeys : 1 << p.page_shift;      // keys of a copy
            const int groups = 1 << (p.page_shift - 3);                         // 8-key rows of a page
            const int32_t none = (int32_t)(p.num_blocks * 2 * groups);          // beyond the cache: zeros
            uint32_t n = 0, st = 0, ph = 1;           // stages filled; the next one and the phase that frees it
            uint32_t is_raw = 0, ph_raw = 0;          // by stage: filled behind `raw`; its last phase
            struct Ahead {                            // a segment as it is loaded
                int kt0, tiles, keys, common, kvh;
                const int32_t *table;
            };
            // this lane's block id of a tile's pages
            auto block = [&](const Ahead &x, int kt) -> int32_t {
                const int first = kt * kKeys + lane * box;
                if (kt >= x.kt0 + x.tiles || lane >= per || first >= x.keys)
                    return -1;
                return x.table[first >> p.page_shift];
            };
            // the next segment, described to the other warps; tiles = -1: there is none
            uint32_t seg = 0;
            auto describe = [&](Ahead &x, int32_t &id) -> bool {
                Info *const info = &sm.info[seg % kRing];
                const bool have = walk.next(s);
                x.tiles = -1;
                if (seg >= kRing && !wait(smem_u32(&sm.info_empty[seg % kRing]), (seg / kRing - 1) & 1))
                    return false;
                if (have) {
                    x.kt0 = s.kt0;
                    x.kvh = s.kvh;
                    x.keys = walk.all_keys(s);
                    x.common = walk.common_keys(s);
                    x.tiles = group_tiles(s, x.keys);
                    x.table = s.b < 0 ? p.prefix_table : p.table + s.b * p.max_pages;
                    id = block(x, x.kt0);             // on its way while the segment is described
                    if (lane < NG) {
                        // a decode step's own items have one tile of rows: the groups have them in turn
                        const bool own_item = Plan::kDecode && s.b >= 0;
                        const int q = NG == 2 && own_item ? lane ^ (int)(seg & 1) : lane;
                        const int r0 = (s.rt * NG + q) * 128, left = s.rows - r0;
                        const int t = s.b < 0 || !Plan::kDecode ? p.by_group.div(r0) : 0;
                        const int own = walk.group_keys(s, q);
                        info->g[lane].head = r0 - t * p.group;
                        info->g[lane].rows = left < 0 ? 0 : left < 128 ? left : 128;
                        info->g[lane].keys = own;
                        info->g[lane].at = own_item ? 0 : lane * 128;
                        info->g[lane].tiles = group_tiles(s, own);
                        if constexpr (Plan::kDecode) {
                            info->g[lane].row0 = s.b < 0 ? t : s.b;
                            info->g[lane].key0 = x.keys;
                        } else {
                            info->g[lane].row0 = plan.req[s.b].row0 + t;
                            info->g[lane].key0 = plan.req[s.b].pos0 + t + 1;
                        }
                    }
                    if (lane == 0) {
                        info->kt0 = s.kt0;
                        info->all = x.keys;
                        info->common = x.common;
                        info->head0 = s.kvh * p.group;
                        int rows = 0;
                        info->slot = s.whole && (!Plan::kDecode || p.prefix_len == 0)
                                         ? -1
                                         : slot_of<D, NG, Plan>(p, s, cta, &rows);
                        info->slot_rows = rows;
                    }
                }
                if (lane == 0)
                    info->most = x.tiles;
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(smem_u32(&sm.info_full[seg % kRing]));
                ++seg;
                return true;
            };
            // a segment is described, and its first block ids requested, behind the first loads of the one in
            // front
            Ahead now, then;
            int32_t id = -1;
            bool go = describe(now, id);
            while (go && now.tiles >= 0) {
                int32_t then_id = -1;
                const int tiles = now.tiles, keys = now.keys, common = now.common;
                for (int j = 0; go && j < (tiles > 0 ? tiles : 1); ++j) {
                    if (j == (tiles > 1 ? 1 : 0)) {
                        go = describe(then, then_id);
                        if (!go)
                            break;
                        if (tiles == 0)
                            break;
                    }
                    const int kt = now.kt0 + j;
                    const int32_t blk = id;
                    id = block(now, kt + 1);          // a tile ahead of its copies
                    const int first = kt * kKeys + lane * box;
                    const bool mine = lane < per && first < keys;
                    const bool good = blk >= 0 && blk < p.num_blocks;
                    if (mine && !good)
                        report(p.d_err, HS_DEVERR_BLOCK_OOB);
                    const int pages = __popc(__ballot_sync(0xffffffffu, mine));
                    const int in_page = (first & ((1 << p.page_shift) - 1)) >> 3;
                    for (int plane = 0; plane < 2; ++plane) {
                        // the first round of waits passes: no phase is over yet
                        if (!wait(empty(st), ph)) {
                            go = false;
                            break;
                        }
                        const bool raw = plane == 1 && (kt + 1) * kKeys > common;
                        const uint32_t bar = raw ? smem_u32(&sm.raw[st]) : full(st);
                        is_raw = raw ? is_raw | 1u << st : is_raw & ~(1u << st);
                        ph_raw ^= raw ? 1u << st : 0u;
                        if (lane == 0)
                            mbar_arrive_expect_tx(bar, (uint32_t)(pages * box * D * 2));
                        __syncwarp();
                        if (mine)
                            tma_load_4d(st_at + st * C::kTile + lane * box * D * 2, &map, 0, 0,
                                        now.kvh * kHalf,
                                        good ? (blk * 2 + plane) * groups + in_page : none, bar);
                        __syncwarp();
                        ++n;
                        if (++st == kSt) {
                            st = 0;
                            ph ^= 1;
                        }
                    }
                }
                now = then;
                id = then_id;
            }
            // the copies and MMAs in flight end (bounded) before their memory goes away
            for (uint32_t i = n > kSt ? n - kSt : 0; i < n; ++i) {
                const uint32_t at = i % kSt;
                if (!wait(empty(at), (i / kSt) & 1)) {
                    if ((is_raw >> at) & 1)
                        mbar_wait_bounded(smem_u32(&sm.raw[at]), ((ph_raw >> at) & 1) ^ 1, kTimeoutNs);
                    else
                        mbar_wait_bounded(full(at), (i / kSt) & 1, kTimeoutNs);
                }
            }
        } else if (warp >= C::kSoftmax && warp < C::kSoftmax + NG) {
            // ---- MMAs, a warp to a group, in the order QK(0), PV(0), QK(1), PV(1), ...: the scores of the
            // next tile overwrite the weights of the last one behind the product that reads them.  A stage
            // is free once both groups are done with it
            const int g = warp - C::kSoftmax;
            const uint32_t s_at = tmem + g * 256, o_at = s_at + 128, p_at = s_at + C::kWeightsAt;
            const uint32_t bar_q = smem_u32(&sm.q_full[g]), bar_s = smem_u32(&sm.s_full[g]);
            const uint32_t bar_p = smem_u32(&sm.p_full[g]), bar_o = smem_u32(&sm.o_full[g]);
            const uint32_t bar_r = smem_u32(&sm.s_read[g]);
            const uint64_t q_desc = sdesc_sw128(q_at + g * C::kTile, 16, 1024);
            const uint64_t k_desc = sdesc_sw128(st_at, 16, kHalf * 1024);
            const uint64_t v_desc = sdesc_sw128(st_at, 1024, kHalf * 1024);
            uint32_t st = 0, ph = 0;         // the stage at hand and the phase of its use
            auto next_stage = [&]() {
                if (++st == kSt) {
                    st = 0;
                    ph ^= 1;
                }
            };
            auto qk = [&]() {                // the scores of the tile at hand; its stage is free behind them
                if (elect_one()) {
                    const uint64_t b = k_desc + st * (C::kTile / 16);
    #pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_f16_ss(s_at, q_desc + ((k >> 2) * 16384 + (k & 3) * 32) / 16,
                                   b + ((k >> 2) * 1024 + (k & 3) * 32) / 16, Elem<T>::idesc(kKeys, 0), k > 0);
                    tc_commit(bar_s);
                    tc_commit(empty(st));
                }
                __syncwarp();
            };
            auto pass = [&]() -> bool {      // a stage that this group has no use for
                if (!wait(full(st), ph))
                    return false;
                if (lane == 0)
                    mbar_arrive(empty(st));
                __syncwarp();
                next_stage();
                return true;
            };
            // the next tile's scores, or its keys left to the other group
            auto next_scores = [&](int j, int mine, int most) -> bool {
                if (j + 1 < mine) {
                    if (!wait(full(st), ph))
                        return false;
                    tc_fence_after();
                    qk();
                    next_stage();
                } else if (j + 1 < most) {
                    return pass();
                }
                return true;
            };
            uint32_t ph_q = 0, ph_p = 0, ph_turn = (uint32_t)g ^ 1;    // the first group has the first turn
            bool go = true;
            if (p.stall_for_test && g == 0)
                go = wait(smem_u32(&sm.drain[0]), 0);     // only this warp commits to it, at the end
            for (uint32_t seg = 0; go; ++seg) {
                go = described(seg);
                if (!go)
                    break;
                const Info &info = sm.info[seg % kRing];
                const int most = info.most, mine = info.g[g].tiles;
                const int both = NG == 2 && !C::kOwnWeights ? min(mine, info.g[(g + 1) % NG].tiles) : 0;
                int left = info.g[g].keys - info.kt0 * kKeys;
                done_with(seg);
                if (most < 0)
                    break;
                if (mine > 0) {
                    go = wait(bar_q, ph_q) && wait(full(st), ph);
                    ph_q ^= 1;
                    if (!go)
                        break;
                    tc_fence_after();
                    qk();
                    next_stage();
                } else if (most > 0) {
                    go = pass();
                }
                for (int j = 0; j < most && go; ++j, left -= kKeys) {
                    if (j >= mine) {
                        go = pass() && (j + 1 == most || pass());
                        continue;
                    }
                    const int steps = left >= kKeys ? kKeys / 16 : (left + 15) / 16;
                    const uint32_t st_v = st, ph_v = ph;
                    if constexpr (C::kOwnWeights) {
                        go = wait(bar_r, ph_p);
                        next_stage();
                        go = go && next_scores(j, mine, most);
                    }
                    go = go && wait(bar_p, ph_p) && wait(full(st_v), ph_v);
                    ph_p ^= 1;
                    // The groups take turns, a product with v and the next scores each.  Where both had their
                    // products in flight at once they ended at once, did their softmax at once and stayed so:
                    // 2.1 us a tile instead of 1.5.
                    if (go && j < both) {
                        go = wait(smem_u32(&sm.turn[g]), ph_turn);
                        ph_turn ^= 1;
                    }
                    if (!go)
                        break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t b = v_desc + st_v * (C::kTile / 16);
    #pragma unroll
                        for (int k = 0; k < kKeys / 16; ++k)
                            if (k < steps)
                                mma_f16_ts(o_at, p_at + k * 8, b + k * 2 * kHalf * 1024 / 16,
                                           Elem<T>::idesc(D, 1), (uint32_t)(j > 0 || k > 0));
                        if (C::kOwnWeights || j + 1 == mine)
                            tc_commit(bar_o);
                        tc_commit(empty(st_v));
                    }
                    __syncwarp();
                    if constexpr (!C::kOwnWeights) {
                        next_stage();
                        go = next_scores(j, mine, most);
                        if (!go)
                            break;
                    }
                    if (j < both) {
                        if (lane == 0)
                            mbar_arrive(smem_u32(&sm.turn[1 - g]));
                        __syncwarp();
                    }
                }
            }
            if (*abort != 0) {
                // the MMAs in flight end (bounded) before their memory goes away
                if (elect_one()) {
                    tc_commit(smem_u32(&sm.drain[g]));
                    mbar_wait_bounded(smem_u32(&sm.drain[g]), 0, kTimeoutNs);
                }
                __syncwarp();
            }
        } else {
            // ---- values at masked places: the warps that are left
            constexpr int kWho = (3 - NG) * 32, kRows = kWho / (D / 8);     // rows that they take at once
            uint32_t st_v = 1, ph_raw = 0;         // the stage of the next value tile
            const int who = tid - (C::kSoftmax + NG) * 32;
            auto pair_and = [](bool x) {
                int r;
                asm volatile("{\n\t.reg .pred p, q;\n\t"
                             "setp.ne.s32 p, %1, 0;\n\t"
                             "bar.red.and.pred q, 1, %2, p;\n\t"
                             "selp.s32 %0, 1, 0, q;\n\t}"
                             : "=r"(r)
                             : "r"((int)x), "n"(kWho)
                             : "memory");
                return r != 0;
            };
            auto pair_sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(kWho) : "memory"); };
            bool go = true;
            for (uint32_t seg = 0; go; ++seg) {
                go = pair_and(described(seg));
                if (!go)
                    break;
                const Info &info = sm.info[seg % kRing];
                const int tiles = info.most, all = info.all, common = info.common, kt0 = info.kt0;
                if (tiles < 0)
                    break;
                int32_t *const any = &sm.marks.any[seg % kRing], *const from = sm.marks.from[seg % kRing];
                bool clean = Plan::kDecode;              // a decode step has no keys that only some rows see
                for (int j = 0; j < tiles; ++j, st_v = (st_v + 2) % kSt) {
                    const int k0 = (kt0 + j) * kKeys;
                    if (k0 + kKeys <= common)
                        continue;
                    if (!clean) {
                        for (int i = who; i < D; i += kWho)
                            from[i] = INT_MAX;
                        if (who == 0)
                            *any = 0;
                        clean = true;
                        pair_sync();
                    }
                    const uint32_t st = st_v;
                    // these warps go on or none: they meet in a plain barrier below
                    go = pair_and(wait(smem_u32(&sm.raw[st]), (ph_raw >> st) & 1));
                    ph_raw ^= 1u << st;
                    if (!go)
                        break;
                    uint8_t *const v = smem_raw + (NG + st) * C::kTile;
                    // rows [common, all) are searched, rows behind them up to a step of the MMA zeroed
                    const int lo = common > k0 ? common - k0 : 0;
                    const int hi = all - k0 < kKeys ? all - k0 : kKeys;
                    const int end = (hi + 15) / 16 * 16;
                    // 16 bytes at a time: chunk x of row r is chunk x & 7 of half x >> 3, swizzled
                    auto chunk = [&](int r, int x) {
                        return reinterpret_cast<uint4 *>(v + ((r >> 3) * kHalf + (x >> 3)) * 1024 +
                                                         (r & 7) * 128 + (((x & 7) ^ (r & 7)) << 4));
                    };
                    const int x = who % (D / 8), r_who = who / (D / 8);
                    for (int r = hi + r_who; r < end; r += kRows)
                        *chunk(r, x) = make_uint4(0, 0, 0, 0);
                    if (lo < hi)
                        pair_sync();
                    // Searched are whole atoms of 8 rows, kRows of them at a time, so that a lane's places in
                    // an atom are constants; a product with zero for two values says whether one is not finite.
                    // (Testing exponents took over 10 us a tile of 128 rows: 8k tokens of 32 heads of their own
                    // 574 us where this took 398.)
                    for (int a0 = lo >> 3; lo < hi && a0 < (hi + 7) >> 3; a0 += kRows) {
                        uint4 y[8];
    #pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int r = (a0 + k * kRows / 8) * 8 + k * kRows % 8 + r_who;
                            y[k] = a0 + k * kRows / 8 < (hi + 7) >> 3 ? *chunk(r, x) : make_uint4(0, 0, 0, 0);
                        }
                        uint32_t z[4] = {0, 0, 0, 0};
    #pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            z[0] = Elem<T>::plus_zero_times(z[0], y[k].x);
                            z[1] = Elem<T>::plus_zero_times(z[1], y[k].y);
                            z[2] = Elem<T>::plus_zero_times(z[2], y[k].z);
                            z[3] = Elem<T>::plus_zero_times(z[3], y[k].w);
                        }
                        if (((z[0] | z[1] | z[2] | z[3]) & 0x7FFF7FFFu) == 0)
                            continue;
                        for (int k = 0; k < 8; ++k) {
                            const int r = a0 * 8 + k * kRows + r_who;
                            if (r < lo || r >= hi)
                                continue;
                            uint16_t *const e = reinterpret_cast<uint16_t *>(chunk(r, x));
                            for (int w = 0; w < 8; ++w)
                                if ((not_finite<T>(e[w]) & 0x8000u) != 0) {
                                    atomicMin(&from[x * 8 + w], k0 + r);
                                    e[w] = 0;
                                    *any = 1;
                                }
                        }
                    }
                    fence_proxy_async_smem();
                    pair_sync();
                    if (who == 0)
                        mbar_arrive(full(st));
                }
                if (go)
                    done_with(seg);
            }
        }
    } else {
        // ---- softmax: thread = row
        more_registers<C::kMoreRegs>();
        const int g = warp >> 2;
        const int r = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + g * 256 + lanes, o_at = s_at + 128, p_at = s_at + C::kWeightsAt;
        const uint32_t bar_q = smem_u32(&sm.q_full[g]), bar_s = smem_u32(&sm.s_full[g]);
        const uint32_t bar_p = smem_u32(&sm.p_full[g]), bar_o = smem_u32(&sm.o_full[g]);
        const uint32_t bar_r = smem_u32(&sm.s_read[g]);
        uint32_t ph_s = 0, ph_o = 0;
        // row x of the group's rows, counted from its first one's token: x / p.group by multiplication,
        // exact for x < 256, p.group <= 128 (the error of the factor is at most p.group, 256 * 128 < 2^16)
        const uint32_t inv_group = 65536u / (uint32_t)p.group + 1;
        auto token_of = [&](int x) { return (int)(((uint32_t)x * inv_group) >> 16); };
        // a warp copies its 32 rows of a segment's queries, a row's 16-byte chunks by neighbouring lanes;
        // what lies in the rows that do not exist reaches no other row
        auto load_q = [&](const Info &x) {
            constexpr int kChunks = D / 8, kRows = 32 / kChunks;
            const int c = lane % kChunks, r0 = (warp & 3) * 32 + lane / kChunks;
            const int first = x.g[g].head + r0, left = x.g[g].rows - r0;
            const uint32_t to = q_at + g * C::kTile + (c >> 3) * 16384 + r0 * 128;
            const T *const from = static_cast<const T *>(p.q) + x.g[g].row0 * p.q_stride +
                                  (x.head0 + first) * D + c * 8;
            const int turn = (int)(p.q_stride - p.group * D);      // from a token's last head to the next
#pragma unroll 2
            for (int i = 0; i < 32; i += kRows)
                if (i < left)
                    cp_async_16(to + i * 128 + (((c & 7) ^ ((r0 + i) & 7)) << 4),
                                from + (int64_t)token_of(first + i) * turn + i * D);
        };
        auto q_done = [&]() {
            cp_async_wait_all();
            fence_proxy_async_smem();
            mbar_arrive(bar_q);
        };
        bool go = described(0);
        int most = go ? sm.info[0].most : -1, tiles = go ? sm.info[0].g[g].tiles : 0;
        if (most > 0 && tiles > 0) {
            load_q(sm.info[0]);
            q_done();
        }
        for (uint32_t seg = 0; go && most >= 0; ++seg) {
            const Info &info = sm.info[seg % kRing];
            const int rows = info.g[g].rows, head = info.g[g].head;
            const int t = token_of(head + r);
            const int keys = Plan::kDecode ? info.g[g].key0 : info.g[g].key0 + t;
            const bool ok = r < rows;
            const bool some = (warp & 3) * 32 < rows;      // the warp has a row
            // the next segment's queries, behind this one's last weights: its last scores are here, so its
            // queries are done with, and the last product runs meanwhile (384 requests at 100 keys 47 us; 53
            // with this in front of the last softmax)
            int next_most = -1, next_tiles = 0;
            auto ahead = [&]() -> bool {
                if (!described(seg + 1))
                    return false;
                const Info &x = sm.info[(seg + 1) % kRing];
                next_most = x.most;
                next_tiles = next_most > 0 ? x.g[g].tiles : 0;
                if (next_tiles > 0)
                    load_q(x);
                return true;
            };
            float m = -INFINITY, l = 0.f;       // m in units of log2, of scaled scores
            float limit = -INFINITY;            // m + kMost
            float shift = 0.f;                  // -m, but 0 without a key and far from zero
            bool far = false;                   // |m| lies beyond kFar
            int valid = keys - info.kt0 * kKeys;   // keys of the row from this tile on
            for (int j = 0; j < tiles; ++j, valid -= kKeys) {
                go = wait(bar_s, ph_s);
                ph_s ^= 1;
                if (!go)
                    break;
                tc_fence_after();
                // the product before this one, where the scores did not wait for it
                bool behind = !C::kOwnWeights || j == 0;
                auto last_product = [&]() {
                    if (!behind) {
                        go = wait(bar_o, ph_o);
                        ph_o ^= 1;
                        tc_fence_after();
                        behind = true;
                    }
                };
                if (!some) {
                    tc_fence_before();
                    if constexpr (C::kOwnWeights)
                        mbar_arrive(bar_r);
                    last_product();
                    if (!go)
                        break;
                    mbar_arrive(bar_p);
                    continue;
                }
                float x[kKeys];
#pragma unroll
                for (int c = 0; c < kKeys; c += 32)
                    tmem_ld32(s_at + c, *reinterpret_cast<float(*)[32]>(&x[c]));
                tmem_wait_ld();
                if constexpr (C::kOwnWeights) {
                    tc_fence_before();
                    mbar_arrive(bar_r);
                }
                if (__any_sync(0xffffffffu, valid < kKeys)) {
#pragma unroll
                    for (int c = 0; c < kKeys; ++c)
                        x[c] = c < valid ? x[c] : -INFINITY;
                }
                float t0 = max3(x[0], x[1], x[2]), t1 = max3(x[3], x[4], x[5]);
                float t2 = max3(x[6], x[7], x[8]), t3 = max3(x[9], x[10], x[11]);
#pragma unroll
                for (int c = 12; c + 7 < kKeys; c += 8) {
                    t0 = max3(t0, x[c], x[c + 1]);
                    t1 = max3(t1, x[c + 2], x[c + 3]);
                    t2 = max3(t2, x[c + 4], x[c + 5]);
                    t3 = max3(t3, x[c + 6], x[c + 7]);
                }
                t0 = max3(t0, x[124], x[125]);
                t1 = max3(t1, x[126], x[127]);
                const float top = max3(t0, t1, fmaxf(t2, t3)) * p.scale_log2;
                const bool up = top > limit;
                if (__any_sync(0xffffffffu, up || far)) {
                    float to = m;
                    if (up) {
                        to = top - Elem<T>::kBelow;
                        limit = to + Elem<T>::kMost;
                        shift = -to;
                        far = ok && fabsf(to) > Elem<T>::kFar;
                    }
                    const bool any_far = __any_sync(0xffffffffu, far);
                    if (__builtin_expect(any_far, 0) && far) {  // where 8 or 15 is half a step of float32 or less
                        to = up && top - to > Elem<T>::kMost ? top : to;
                        limit = to + Elem<T>::kMost;
                        limit = limit - to > Elem<T>::kMost ? to : limit;
                        shift = 0.f;
                    }
                    const float f = up ? ex2(m - to) : 1.f;
                    m = to;
                    if (j > 0) {
                        // the previous product is done: the scores came after it, or it is waited for
                        last_product();
                        l *= f;
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {      // few registers: the scores hold theirs
                            uint32_t a[16];
                            tmem_ld16(o_at + c, a);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                a[i] = __float_as_uint(__uint_as_float(a[i]) * f);
                            tmem_st16(o_at + c, a);
                        }
                    }
                    // Far from zero the scores are rounded before m is taken off, as their maximum was, and
                    // what is left of them is brought back to the scale of the others.  In a loop of 16
                    // columns, through the columns of the weights, which are free by now: code that hardly
                    // any call runs makes the others wait for theirs (as straight code, two 8k-token prompts
                    // of 64-wide heads 546 us, so 528; 519 without).  Not in pairs: a product and a sum of
                    // two float32 each become one fused instruction.
                    if (__builtin_expect(any_far, 0)) {
                        const float by = far ? p.scale_log2 : 1.f, off = far ? m : 0.f, back = 1.f / by;
                        constexpr int kPart = C::kOwnWeights ? 64 : 128;
#pragma unroll
                        for (int h = 0; h < kKeys; h += kPart) {
#pragma unroll
                            for (int c = 0; c < kPart; c += 16)
                                tmem_st16(p_at + c, *reinterpret_cast<uint32_t(*)[16]>(&x[h + c]));
                            tmem_wait_st();
#pragma unroll 1
                            for (int c = 0; c < kPart; c += 16) {
                                uint32_t a[16];
                                tmem_ld16(p_at + c, a);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    a[i] = __float_as_uint(
                                        __fsub_rn(__fmul_rn(__uint_as_float(a[i]), by), off) * back);
                                tmem_st16(p_at + c, a);
                            }
                            tmem_wait_st();
#pragma unroll
                            for (int c = 0; c < kPart; c += 32)
                                tmem_ld32(p_at + c, *reinterpret_cast<float(*)[32]>(&x[h + c]));
                            tmem_wait_ld();
                        }
                    }
                }
                const uint64_t scale2 = pair(p.scale_log2, p.scale_log2), shift2 = pair(shift, shift);
                uint64_t l01 = 0, l23 = 0;
#pragma unroll
                for (int c = 0; c < kKeys; c += 32) {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const int e = c + 2 * i;
                        const float2 y0 = unpair(fma2(pair(x[e], x[e + 1]), scale2, shift2));
                        const float2 y1 = unpair(fma2(pair(x[e + 2], x[e + 3]), scale2, shift2));
                        const float a0 = ex2(y0.x), a1 = ex2(y0.y), a2 = ex2(y1.x), a3 = ex2(y1.y);
                        l01 = add2(l01, pair(a0, a1));
                        l23 = add2(l23, pair(a2, a3));
                        w[i] = Elem<T>::pack(a0, a1);
                        w[i + 1] = Elem<T>::pack(a2, a3);
                    }
                    if (c == 0)
                        last_product();
                    tmem_st16(p_at + c / 2, w);
                }
                if (!go)
                    break;
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar_p);
                const float2 ls = unpair(add2(l01, l23));
                l += ls.x + ls.y;
            }
            if (!go)
                break;
            go = ahead();
            if (go && tiles > 0) {
                go = wait(bar_o, ph_o);
                ph_o ^= 1;
            }
            if (!go)
                break;
            tc_fence_after();
            if (next_tiles > 0)
                q_done();
            const int last = info.kt0 + tiles;             // behind the group's last tile here
            const bool marked = !Plan::kDecode && tiles > 0 && last * kKeys > info.common &&
                                *(volatile int32_t *)&sm.marks.any[seg % kRing] != 0;
            const int32_t *const from = sm.marks.from[seg % kRing];
            const int row = info.g[g].row0 + t, head_at = info.head0 + head + r - t * p.group;
            const int64_t slot_at = info.slot;
            // 32 columns of the sums.  The loops over them stay loops: straight code that is run once a
            // segment waits for its instructions (a segment's outputs took 2 us of it, as a loop 1.2)
            auto columns = [&](int c, float (&a)[32]) {
                if (tiles > 0) {
                    tmem_ld32(o_at + c, a);
                    tmem_wait_ld();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        a[i] = 0.f;
                }
                if (marked) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        a[i] = keys > from[c + i] ? NAN : a[i];
                }
            };
            if (!some) {
                // nothing to write
            } else if (slot_at < 0) {
                const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
                // four lanes turn their four 16-byte chunks of four rows round, so that a store covers
                // 64 bytes of a row instead of 16
                T *o[4];
                bool on[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int rr = (r & ~3) + k, tt = token_of(head + rr);
                    on[k] = rr < rows;
                    o[k] = static_cast<T *>(p.o) + (info.g[g].row0 + tt) * p.o_stride +
                           (info.head0 + head + rr - tt * p.group) * D + (lane & 3) * 8;
                }
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    float a[32];
                    columns(c, a);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        a[i] = Elem<T>::in_range(a[i] * inv);
                    uint4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int i = 8 * k;
                        v[k] = make_uint4(Elem<T>::pack(a[i], a[i + 1]), Elem<T>::pack(a[i + 2], a[i + 3]),
                                          Elem<T>::pack(a[i + 4], a[i + 5]), Elem<T>::pack(a[i + 6], a[i + 7]));
                    }
                    swap_chunks(v[0], v[1], lane & 1, 1);
                    swap_chunks(v[2], v[3], lane & 1, 1);
                    swap_chunks(v[0], v[2], lane & 2, 2);
                    swap_chunks(v[1], v[3], lane & 2, 2);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (on[k])
                            *reinterpret_cast<uint4 *>(o[k] + c) = v[k];
                }
                if (ok && p.lse != nullptr)
                    p.lse[(int64_t)row * p.n_heads + head_at] =
                        l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
            } else {
                float *const slot = p.part + slot_at;
                const int at = info.g[g].at + r, slot_rows = info.slot_rows;
                if (ok)
                    reinterpret_cast<float2 *>(slot)[at] = make_float2(m, l);
#pragma unroll 1
                for (int c = 0; tiles > 0 && c < D; c += 32) {
                    float a[32];
                    columns(c, a);
                    if (ok && !Plan::kDecode) {
                        float *const to = slot + pairs_floats(128 * NG) + c * 128 * NG + at;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            to[i * 128 * NG] = a[i];
                    } else if (ok) {
                        float *const to = slot + pairs_floats(slot_rows) + (int64_t)at * D + c;
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            *reinterpret_cast<float4 *>(to + i) =
                                make_float4(a[i], a[i + 1], a[i + 2], a[i + 3]);
                    }
                }
            }
            tc_fence_before();
            done_with(seg);
            most = next_most;
            tiles = next_tiles;
        }
        cp_async_wait_all();     // none is left but after a wait that ran out
    }
    tc_fence_before();
    __syncthreads();
    if (*abort != 0 && tid == 0)
        report(p.d_err, HS_DEVERR_TIMEOUT);
    if (warp == C::kSoftmax) {
        tc_fence_after();
        tmem_dealloc(tmem, C::kTmemCols);
    }
}

// ---- joining partial results ---------------------------------------------------------------
//
// With M = max m_i over the parts of a row: o = sum 2^(m_i - M) a_i / L, L = sum 2^(m_i - M) l_i,
// lse = ln 2 (M + log2 L).  One to eight warps take a row, D / 32 columns a lane; warp y of w has
// the parts y, y + w, ..., and their sums are added in the order of the warps, so that the same split
// gives the same bits.  A lane looks up one part's pair and address, so that neither these loads nor
// those of the parts' rows wait for one another: what bounds the join of a few rows is latency.

constexpr int kMergeWarps = 8;

template <int D>
struct Joined {
    float a[D / 32];
    float m, l;
};

// `part(i, pair, a)`: where part i has the row's pair and its a, false if it has none (its CTA has no
// units)
template <int D, typename F>
__device__ __forceinline__ Joined<D> join_parts(const float *base, int count, int first, int step,
                                                int lane, F part)
{
    constexpr int E = D / 32;
    Joined<D> x;
    x.m = -INFINITY;
    x.l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e)
        x.a[e] = 0.f;
    auto rows_of = [&](unsigned there, int64_t at_a, int j0, float (&v)[8][E]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t at = __shfl_sync(0xffffffffu, at_a, j0 + j);
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[j][e] = 0.f;
            if ((there >> (j0 + j)) & 1) {
                if constexpr (E == 4) {
                    const float4 y = *reinterpret_cast<const float4 *>(base + at + lane * 4);
                    v[j][0] = y.x, v[j][1] = y.y, v[j][2] = y.z, v[j][3] = y.w;
                } else {
                    const float2 y = *reinterpret_cast<const float2 *>(base + at + lane * 2);
                    v[j][0] = y.x, v[j][1] = y.y;
                }
            }
        }
    };
    for (int i0 = first; i0 < count; i0 += 32 * step) {
        const int i = i0 + lane * step;
        int64_t at_pair = 0, at_a = 0;
        float2 ml = make_float2(-INFINITY, 0.f);
        const bool here = i < count && part(i, at_pair, at_a);
        if (here)
            ml = *reinterpret_cast<const float2 *>(base + at_pair);
        const unsigned there = __ballot_sync(0xffffffffu, here);
        const int last = 32 - __clz(there);
        float v[8][E];
        rows_of(there, at_a, 0, v);
        // a part without a key of this row: what it holds of a means nothing
        const bool live = !(ml.x == -INFINITY && ml.y == 0.f);
        float top = ml.x;
#pragma unroll
        for (int w = 16; w > 0; w >>= 1)
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
        top = fmaxf(top, x.m);
        const float f = x.m == -INFINITY && x.l == 0.f ? 0.f : ex2(x.m - top);
        const float h = live ? ex2(ml.x - top) : 0.f;
        float l = live ? ml.y * h : 0.f;
#pragma unroll
        for (int w = 16; w > 0; w >>= 1)
            l += __shfl_xor_sync(0xffffffffu, l, w);
        x.m = top;
        x.l = x.l * f + l;
#pragma unroll
        for (int e = 0; e < E; ++e)
            x.a[e] *= f;
        const unsigned any = __ballot_sync(0xffffffffu, live);
        for (int j0 = 0; j0 < last; j0 += 8) {
            if (j0 > 0)
                rows_of(there, at_a, j0, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float hj = __shfl_sync(0xffffffffu, h, j0 + j);
                if ((any >> (j0 + j)) & 1) {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        x.a[e] = fmaf(v[j][e], hj, x.a[e]);
                }
            }
        }
    }
    return x;
}

template <typename T, int D>
__device__ __forceinline__ void write_row(const AttnParams &p, const Joined<D> &x, int64_t row, int head,
                                          int lane)
{
    const float inv = x.l > 0.f ? 1.f / x.l : (x.l == 0.f ? 0.f : x.l);
    uint32_t *o = reinterpret_cast<uint32_t *>(static_cast<T *>(p.o) + row * p.o_stride + head * D +
                                               lane * (D / 32));
#pragma unroll
    for (int i = 0; i < D / 32; i += 2)
        o[i / 2] = Elem<T>::pack(Elem<T>::in_range(x.a[i] * inv), Elem<T>::in_range(x.a[i + 1] * inv));
    if (p.lse != nullptr && lane == 0)
        p.lse[row * p.n_heads + head] = x.l == 0.f ? -INFINITY : kLn2 * (x.m + log2f(x.l));
}

// the warps of a row join their sums and the first of them writes the row (all threads of the block
// call this; `on`: the row exists)
template <typename T, int D>
__device__ __forceinline__ void finish_row(const AttnParams &p, Joined<D> x, int per_row, int warp,
                                           int lane, bool on, int64_t row, int head)
{
    __shared__ float sums[kMergeWarps][D + 2];
    constexpr int E = D / 32;
    if (per_row > 1) {
        float *const own = sums[warp];
#pragma unroll
        for (int e = 0; e < E; ++e)
            own[lane * E + e] = x.a[e];
        if (lane == 0) {
            own[D] = x.m;
            own[D + 1] = x.l;
        }
        __syncthreads();
        if (warp % per_row == 0) {
            float top = x.m;
            for (int w = 1; w < per_row; ++w)
                top = fmaxf(top, sums[warp + w][D]);
            float l = 0.f, a[E];
#pragma unroll
            for (int e = 0; e < E; ++e)
                a[e] = 0.f;
            for (int w = 0; w < per_row; ++w) {
                const float *const from = sums[warp + w];
                if (from[D] == -INFINITY && from[D + 1] == 0.f)
                    continue;
                const float h = ex2(from[D] - top);
                l += from[D + 1] * h;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    a[e] = fmaf(from[lane * E + e], h, a[e]);
            }
            x.m = top;
            x.l = l;
#pragma unroll
            for (int e = 0; e < E; ++e)
                x.a[e] = a[e];
        }
        __syncthreads();
    }
    if (on && warp % per_row == 0)
        write_row<T, D>(p, x, row, head, lane);
}

// ---- launch --------------------------------------------------------------------------------

// The cache of a layer as [8-token group][64-element block of a token's heads][token][64]: a copy's
// box is one head of a page (or of 128 keys of one), 8-token groups outermost, which in shared
// memory is the operand layout of both products: 128-byte rows, swizzled, in atoms of 8 tokens, the
// atoms of a row's blocks side by side.  Misses fetch 128 bytes: with 256 the neighbour's head of 64 came
// along for nothing (64 decode steps of 8 such heads at 4,096 keys 126 us instead of 96).
template <int D>
bool encode_cache(CUtensorMap *m, const AttnParams &p)
{
    auto fn = encode_fn();
    if (fn == nullptr)
        return false;
    const uint64_t page = 1ull << p.page_shift, row = (uint64_t)p.n_kv * D;
    cuuint64_t dim[4] = {64, 8, row / 64, (uint64_t)p.num_blocks * 2 * page / 8};
    cuuint64_t stride[3] = {row * 2, 128, 8 * row * 2};
    cuuint32_t box[4] = {64, 8, D / 64, (cuuint32_t)((page < kKeys ? page : kKeys) / 8)};
    cuuint32_t one[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, const_cast<void *>(p.cache), dim, stride, box, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, int NG, class Plan>
cudaError_t launch_tc(const AttnParams &p, const Plan &plan, cudaStream_t s)
{
    CUtensorMap map;
    if (!encode_cache<D>(&map, p))
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> smem_set{0};
    return launch_pdl_big_smem(attn_kernel<T, D, NG, Plan>, dim3((unsigned)p.ctas),
                               dim3(Cfg<D, NG>::kThreads), smem_bytes<D, NG>(), s, smem_set, p, plan, map);
}

}  // namespace attn
}  // namespace hs
