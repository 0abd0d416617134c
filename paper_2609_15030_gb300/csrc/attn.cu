// Softmax attention over the paged cache (the full-attention layers) on tcgen05 tensor cores.
//
// Rows.  The query heads of one KV head are stacked: row r of an item is token r / group, head
// r % group, so that one tile of keys serves all of them.  An item is NG tiles of 128 rows of one
// (request, KV head); its keys are walked in tiles of 128.  The units of work are (item, key tile).
//
// Mathematics, per row, with s_j = scale * log2(e) * q . k_j:  m is a number near max s_j,
// l = sum 2^(s_j - m), a = sum 2^(s_j - m) v_j, all float32;  o = a / l, lse = ln 2 (m + log2 l).
// m follows the maximum lazily: only when a tile's maximum exceeds it by more than 8 are l and a
// rescaled by 2^(m_old - m_new) (weights then reach 2^8 at most, and nothing is lost: the scale
// of 16-bit weights is free).  Weights are rounded to the element type for the product with v (the
// tensor core takes 16-bit operands); l sums them before that rounding.
//
// Schedule.  The units of all items in order are shared out evenly over the CTAs, each a
// contiguous run, so that one long request or many ragged ones fill the SMs alike.  An item whose
// keys fall to several CTAs leaves (m, l, a) of each in the workspace and attn_merge_kernel joins
// them.  With `unsplit` a CTA takes the whole items that begin in its run.
//
// Warps.  Per tile of rows one group of four softmax warps (thread = row = TMEM lane), then one
// warp that issues the MMAs, one that loads keys and values by TMA, one that looks after values at
// masked places.  Per key tile and group: S = Q K^T into TMEM; the group reads it, writes the
// weights over it as 16-bit pairs; O += P V with P as the TMEM operand.  With two groups the
// tensor core works on one while the other is in its softmax.
//
// Values at masked places.  A weight of zero times a NaN or an infinity is NaN, so v must be finite
// wherever some row of the tile does not attend: rows behind the last key are zeroed in shared
// memory, and keys that only some rows see (the causal diagonal) are searched; a value there that
// is not finite is zeroed and noted, and the rows that do see it get NaN in its column at the end.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>

#include "attn_internal.cuh"
#include "sm100_ptx.cuh"

namespace hs {
namespace {

using namespace ptx;

constexpr int kKeys = 128;               // keys per tile
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.0f;            // log2 of the largest weight
constexpr uint64_t kTimeoutNs = 1000000000ull;

// ---- shapes of a launch --------------------------------------------------------------------

template <int D, int NG>
struct Cfg {
    static constexpr int kTile = kKeys * D * 2;            // bytes of a tile of keys, values or rows
    // two groups: one CTA per SM, as many stages as fit; one group: two CTAs per SM
    static constexpr int kStages = NG == 2 ? (D == 128 ? 5 : 8) : (D == 128 ? 2 : 5);
    // segments whose notes on values are kept.  A value tile is searched once the stage it lies in
    // is free of the tile kStages / 2 before; the MMAs of that tile's segment began after both
    // groups had left the segment before the one before it
    static constexpr int kMarks = kStages <= 5 ? 4 : 8;
    static constexpr int kSoftmax = NG * 4;                // warps
    static constexpr int kThreads = (kSoftmax + 4) * 32;   // the last warp only lends its registers
    // registers of a softmax thread and of another one, out of those of the launch (65,536 over the
    // resident threads, a multiple of 8): 256 x 224 + 128 x 56 = 384 x 168 and
    // 128 x 200 + 128 x 56 = 256 x 128
    static constexpr int kRegs = NG == 2 ? 168 : 128;
    static constexpr int kMoreRegs = NG == 2 ? 224 : 200, kLessRegs = 56;
    static_assert(kSoftmax * 32 * kMoreRegs + 128 * kLessRegs <= kThreads * kRegs, "");
    static constexpr int kTmemCols = NG == 2 ? 512 : 256;  // S and O of each group, 128 columns each
};

// where a CTA's run of units begins and ends
struct Start {
    int64_t u, u1;
    int32_t b, rt, kvh, kt;
};

// shared memory behind the tiles
template <int D, int NG>
struct Smem {
    uint64_t full[8], empty[8];          // a stage may be read / its MMAs are done
    uint64_t raw[8];                     // a value tile with masked places has landed
    uint64_t q_full[2], s_full[2], p_full[2], o_full[2];
    uint64_t drain;
    uint32_t tmem;
    int32_t abort;
    Start start;
    union {
        int32_t len[HS_MAX_BATCH];       // decode: keys, or -1 for a length out of bounds
        struct {                         // prefill: values that are not finite, by segment
            int32_t any[Cfg<D, NG>::kMarks];
            int32_t from[Cfg<D, NG>::kMarks][D];   // first such position in the column
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

// ---- the walk over items -------------------------------------------------------------------

__host__ __device__ __forceinline__ int tiles_of(int keys)
{
    return (keys + kKeys - 1) / kKeys;
}

__host__ __device__ __forceinline__ int64_t first_unit(int64_t units, int ctas, int c)
{
    return units * c / ctas;
}

// the CTA that has unit u: the largest c with first_unit(c) <= u
__device__ __forceinline__ int cta_of(int64_t units, int ctas, int64_t u)
{
    return (int)(((u + 1) * ctas - 1) / units);
}

__device__ __forceinline__ bool has_units(int64_t units, int ctas, int c)
{
    return first_unit(units, ctas, c) < first_unit(units, ctas, c + 1);
}

// b = -1 stands for the shared prefix, whose rows are those of all requests
template <int NG>
__host__ __device__ __forceinline__ int row_tiles(int rows)
{
    return (rows + 128 * NG - 1) / (128 * NG);
}

// prefill: key tiles of a request's row tile
template <int NG>
__host__ __device__ __forceinline__ int prefill_tiles(int pos0, int n_tokens, int group, int rt)
{
    const int64_t last = ((int64_t)(rt + 1) * 128 * NG - 1) / group;
    return tiles_of(pos0 + (int)(last < n_tokens - 1 ? last : n_tokens - 1) + 1);
}

// one item's key tiles [kt0, kt1) as one CTA has them
struct Segment {
    int b, rt, kvh, kt0, kt1;
    int rows;        // of the whole request (or of all, for the prefix)
    bool whole;      // all of the item's key tiles
    int item;        // running number of the item within its part (prefix or requests), decode only
};

template <int NG>
struct Walk {
    const AttnParams &p;
    const int32_t *len;
    int64_t u, u1;
    int b, rt, kvh, kt;

    __device__ int rows() const
    {
        return b < 0 ? p.batch * p.group : p.kv_len != nullptr ? p.group : p.n_tokens[b] * p.group;
    }
    __device__ int tiles() const
    {
        if (b < 0)
            return tiles_of(p.prefix_len);
        if (p.kv_len != nullptr)
            return len[b] > 0 ? tiles_of(len[b]) : 1;   // an empty row is written by someone
        return prefill_tiles<NG>(p.pos0[b], p.n_tokens[b], p.group, rt);
    }
    __device__ bool skip() const
    {
        return p.kv_len != nullptr ? len[b] < 0 : p.n_tokens[b] == 0;
    }
    __device__ void next_item()
    {
        kt = 0;
        if (++kvh < p.n_kv)
            return;
        kvh = 0;
        if (++rt < row_tiles<NG>(rows()))
            return;
        rt = 0;
        do
            ++b;
        while (b < p.batch && skip());
    }
    __device__ Walk(const AttnParams &params, const int32_t *lens, const Start &s)
        : p(params), len(lens), u(s.u), u1(s.u1), b(s.b), rt(s.rt), kvh(s.kvh), kt(s.kt)
    {
        if (p.unsplit && u < u1 && kt != 0) {         // begins with the next whole item
            u += tiles() - kt;
            next_item();
        }
    }
    __device__ bool next(Segment &s)
    {
        if (u >= u1)
            return false;
        const int n = tiles();
        int take = n - kt;
        if (!p.unsplit && take > u1 - u)
            take = (int)(u1 - u);
        s.b = b;
        s.rt = rt;
        s.kvh = kvh;
        s.kt0 = kt;
        s.kt1 = kt + take;
        s.rows = rows();
        s.whole = kt == 0 && take == n;
        s.item = (b < 0 ? rt : b) * p.n_kv + kvh;
        u += take;
        kt += take;
        if (kt == n)
            next_item();
        return true;
    }
};

// keys that the last row of group g of a segment's row tile attends to (0: the group has no row)
template <int NG>
__device__ __forceinline__ int group_keys(const AttnParams &p, const int32_t *len, const Segment &s,
                                          int g)
{
    const int r0 = (s.rt * NG + g) * 128;
    if (r0 >= s.rows)
        return 0;
    if (s.b < 0)
        return p.prefix_len;
    if (p.kv_len != nullptr)
        return len[s.b];
    const int last = (s.rows - r0 < 128 ? s.rows : r0 + 128) - 1;
    return p.pos0[s.b] + last / p.group + 1;
}

// keys that every row of the segment's item attends to
template <int NG>
__device__ __forceinline__ int common_keys(const AttnParams &p, const int32_t *len, const Segment &s)
{
    if (s.b < 0)
        return p.prefix_len;
    if (p.kv_len != nullptr)
        return len[s.b];
    return p.pos0[s.b] + s.rt * 128 * NG / p.group + 1;
}

// tiles of the segment that a group with `keys` keys takes part in
__device__ __forceinline__ int group_tiles(const Segment &s, int keys)
{
    const int n = tiles_of(keys);
    const int end = n < s.kt1 ? n : s.kt1;
    return end > s.kt0 ? end - s.kt0 : 0;
}

// decode: units of request b (0: its length is out of bounds and it is skipped)
__device__ __forceinline__ int own_units(const AttnParams &p, int len)
{
    return len < 0 ? 0 : (len > 0 ? tiles_of(len) : 1) * p.n_kv;
}

__device__ __forceinline__ int warp_scan(int x, int lane)
{
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, w);
        if (lane >= w)
            x += y;
    }
    return x;
}

// decode, one warp: the lengths into shared memory; returns the units of all requests, and in
// *before those of the requests in front of `upto`
__device__ __forceinline__ int read_lengths(const AttnParams &p, int32_t *len, int lane, bool complain,
                                            int upto, int *before)
{
    int sum = 0, part = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const int b = b0 + lane;
        int n = -1;
        if (b < p.batch) {
            n = p.kv_len[b];
            if (n < 0 || n > p.max_kv) {
                if (complain)
                    report(p.d_err, HS_DEVERR_LENGTH);
                n = -1;
            }
            len[b] = n;
        }
        const int x = own_units(p, n);
        sum += x;
        part += b < upto ? x : 0;
    }
    __syncwarp();
    *before = __reduce_add_sync(0xffffffffu, part);
    return __reduce_add_sync(0xffffffffu, sum);
}

// where CTA c's run begins (one warp; decode: with the lengths in shared memory, `own` their units)
template <int NG>
__device__ __forceinline__ Start find_start(const AttnParams &p, const int32_t *len, int own, int c,
                                            int lane)
{
    Start s;
    if (p.kv_len == nullptr) {
        s.u = first_unit(p.units, p.ctas, c);
        s.u1 = first_unit(p.units, p.ctas, c + 1);
        s.b = p.start_b[c];
        s.rt = p.start_item[c] / p.n_kv;
        s.kvh = p.start_item[c] - s.rt * p.n_kv;
        s.kt = p.start_kt[c];
        return s;
    }
    const int per = tiles_of(p.prefix_len);
    const int pre = per * p.n_kv * row_tiles<NG>(p.batch * p.group);
    const int64_t units = (int64_t)pre + own;
    s.u = first_unit(units, p.ctas, c);
    s.u1 = first_unit(units, p.ctas, c + 1);
    s.b = -1;
    s.rt = s.kvh = s.kt = 0;
    if (s.u < pre) {
        const int item = (int)s.u / per;
        s.kt = (int)s.u - item * per;
        s.rt = item / p.n_kv;
        s.kvh = item - s.rt * p.n_kv;
        return s;
    }
    int v = (int)(s.u - pre);                 // the request with unit v of all requests'
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const int b = b0 + lane;
        const int x = own_units(p, b < p.batch ? len[b] : -1);
        const int incl = warp_scan(x, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, v < incl);
        const int last = __shfl_sync(0xffffffffu, incl, 31);
        if (hit != 0) {
            const int at = __ffs(hit) - 1;
            v -= __shfl_sync(0xffffffffu, incl - x, at);
            s.b = b0 + at;
            const int n = len[s.b] > 0 ? tiles_of(len[s.b]) : 1;
            s.kvh = v / n;
            s.kt = v - s.kvh * n;
            return s;
        }
        v -= last;
    }
    return s;                                 // no unit is left: s.u == s.u1
}

// ---- partial results -----------------------------------------------------------------------
//
// A slot holds R rows: R pairs (m, l), padded to 16 bytes, then R rows of D floats a.  Without a shared prefix an item
// leaves a partial result in at most two places of a CTA's run: at its beginning, where it does not
// start the item (slot 2 cta), and at its end, where it does (slot 2 cta + 1).  Behind a shared
// prefix every segment is partial; its slot is item + cta, which no other segment of its part
// (prefix, requests) has, since both only grow along the run.

__host__ __device__ __forceinline__ int pairs_floats(int rows)
{
    return (2 * rows + 3) / 4 * 4;
}

template <int D>
__host__ __device__ __forceinline__ int64_t slot_floats(int rows)
{
    return pairs_floats(rows) + (int64_t)rows * D;
}

template <int D, int NG>
__host__ __device__ __forceinline__ int64_t prefix_part_floats(const AttnParams &p)
{
    return (int64_t)(row_tiles<NG>(p.batch * p.group) * p.n_kv + p.ctas) * slot_floats<D>(128 * NG);
}

// rows of a slot of the requests' part: an item's
template <int NG>
__host__ __device__ __forceinline__ int slot_rows(const AttnParams &p)
{
    return p.kv_len != nullptr ? p.group : 128 * NG;
}

template <int D, int NG>
__device__ __forceinline__ float *slot_of(const AttnParams &p, const Segment &s, int cta, int *rows)
{
    if (s.b < 0) {
        *rows = 128 * NG;
        return p.part + (int64_t)(s.item + cta) * slot_floats<D>(128 * NG);
    }
    *rows = slot_rows<NG>(p);
    if (p.prefix_len > 0)
        return p.part + prefix_part_floats<D, NG>(p) + (int64_t)(s.item + cta) * slot_floats<D>(*rows);
    return p.part + (int64_t)(2 * cta + (s.kt0 == 0)) * slot_floats<D>(*rows);
}

// ---- element types -------------------------------------------------------------------------

template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
    static constexpr uint32_t kExp = 0x7F807F80u, kOne = 0x00800080u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static constexpr uint32_t idesc(int N, int mn) { return idesc_bf16(128, N, mn); }
};
template <>
struct Elem<__half> {
    static constexpr uint32_t kExp = 0x7C007C00u, kOne = 0x04000400u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static constexpr uint32_t idesc(int N, int mn) { return idesc_f16(128, N, mn); }
};

// sign bits of the 16-bit halves whose exponent is all ones (infinities and NaN)
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x)
{
    return ((x & Elem<T>::kExp) + Elem<T>::kOne) & 0x80008000u;
}

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// ---- the kernel ----------------------------------------------------------------------------

template <typename T, int D, int NG>
__global__ void __launch_bounds__(Cfg<D, NG>::kThreads, NG == 2 ? 1 : 2)
attn_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap map)
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
                if (globaltimer_ns() - t0 > kTimeoutNs)
                    *abort = 1;
            }
        }
        return __all_sync(0xffffffffu, ok);
    };

    if (tid == 0) {
        for (int i = 0; i < kSt; ++i) {
            mbar_init(full(i), 1);
            mbar_init(empty(i), 1);
            mbar_init(smem_u32(&sm.raw[i]), 1);
        }
        for (int g = 0; g < NG; ++g) {
            mbar_init(smem_u32(&sm.q_full[g]), 128);
            mbar_init(smem_u32(&sm.s_full[g]), 1);
            mbar_init(smem_u32(&sm.p_full[g]), 128);
            mbar_init(smem_u32(&sm.o_full[g]), 1);
        }
        mbar_init(smem_u32(&sm.drain), 1);
        fence_mbar_init();
        sm.abort = 0;
    }
    if (warp == C::kSoftmax)
        tmem_alloc(smem_u32(&sm.tmem), C::kTmemCols);
    pdl_wait();
    if (warp == C::kSoftmax + 1) {
        int before = 0;
        const int own = p.kv_len != nullptr ? read_lengths(p, sm.len, lane, cta == 0, 0, &before) : 0;
        const Start st = find_start<NG>(p, sm.len, own, cta, lane);
        if (lane == 0)
            sm.start = st;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t *)&sm.tmem;
    Walk<NG> walk(p, sm.len, sm.start);
    Segment s;

    if (warp >= C::kSoftmax) {
    fewer_registers<C::kLessRegs>();
    if (warp == C::kSoftmax + 1) {
        // ---- loads: key and value tiles in turn through the stages
        const int per = p.page_shift >= 7 ? 1 : kKeys >> p.page_shift;      // pages of a tile
        const int box = p.page_shift >= 7 ? kKeys : 1 << p.page_shift;      // keys of a copy
        const int groups = 1 << (p.page_shift - 3);                         // 8-key rows of a page
        const int32_t none = (int32_t)(p.num_blocks * 2 * groups);          // beyond the cache: zeros
        uint32_t n = 0;                                                     // stages filled
        uint32_t is_raw = 0, ph_raw = 0;          // by stage: filled behind `raw`; its last phase
        bool go = true;
        while (go && walk.next(s)) {
            int keys = group_keys<NG>(p, sm.len, s, NG - 1);
            if (NG == 2 && keys == 0)
                keys = group_keys<NG>(p, sm.len, s, 0);
            const int tiles = group_tiles(s, keys);
            const int common = common_keys<NG>(p, sm.len, s);
            const int32_t *const table = s.b < 0 ? p.prefix_table : p.table + s.b * p.max_pages;
            // block ids a tile ahead of their copies
            auto block = [&](int kt) -> int32_t {
                const int first = kt * kKeys + lane * box;
                if (lane >= per || first >= keys)
                    return -1;
                return table[first >> p.page_shift];
            };
            int32_t ahead = tiles > 0 ? block(s.kt0) : -1;
            for (int j = 0; j < tiles && go; ++j) {
                const int kt = s.kt0 + j;
                const int32_t blk = ahead;
                if (j + 1 < tiles)
                    ahead = block(kt + 1);
                const int first = kt * kKeys + lane * box;
                const bool mine = lane < per && first < keys;
                const bool good = blk >= 0 && blk < p.num_blocks;
                if (mine && !good)
                    report(p.d_err, HS_DEVERR_BLOCK_OOB);
                const int pages = __popc(__ballot_sync(0xffffffffu, mine));
                const int in_page = (first & ((1 << p.page_shift) - 1)) >> 3;
                for (int plane = 0; plane < 2; ++plane, ++n) {
                    const int st = n % kSt;
                    if (n >= kSt && !wait(empty(st), (n / kSt - 1) & 1)) {
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
                                    s.kvh * kHalf,
                                    good ? (blk * 2 + plane) * groups + in_page : none, bar);
                    __syncwarp();
                }
            }
        }
        // the copies and MMAs in flight end (bounded) before their memory goes away
        for (uint32_t i = n > kSt ? n - kSt : 0; i < n; ++i) {
            const uint32_t st = i % kSt;
            if (!wait(empty(st), (i / kSt) & 1)) {
                if ((is_raw >> st) & 1)
                    mbar_wait_bounded(smem_u32(&sm.raw[st]), ((ph_raw >> st) & 1) ^ 1, kTimeoutNs);
                else
                    mbar_wait_bounded(full(st), (i / kSt) & 1, kTimeoutNs);
            }
        }
    } else if (warp == C::kSoftmax) {
        // ---- MMAs.  Per group the order QK(0), PV(0), QK(1), PV(1), ...: the scores of the next
        // tile overwrite the weights of the last one behind the product that reads them
        uint32_t n = 0;                  // key tiles done: tile i is in stages 2 i and 2 i + 1
        uint32_t ph_q = 0, ph_p[2] = {0, 0};
        bool go = true;
        while (go && walk.next(s)) {
            int keys[2] = {0, 0}, cnt[2] = {0, 0};
            for (int g = 0; g < NG; ++g) {
                keys[g] = group_keys<NG>(p, sm.len, s, g);
                cnt[g] = group_tiles(s, keys[g]);
            }
            const int most = cnt[1] > cnt[0] ? cnt[1] : cnt[0];
            auto qk = [&](int g, uint32_t tile) {
                const uint32_t k_at = st_at + (2 * tile % kSt) * C::kTile;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_f16_ss(tmem + g * 256,
                                   sdesc_sw128(q_at + g * C::kTile + (k >> 2) * 16384 + (k & 3) * 32, 16,
                                               1024),
                                   sdesc_sw128(k_at + (k >> 2) * 1024 + (k & 3) * 32, 16, kHalf * 1024),
                                   Elem<T>::idesc(kKeys, 0), k > 0);
                    tc_commit(smem_u32(&sm.s_full[g]));
                }
                __syncwarp();
            };
            for (int j = 0; j < most && go; ++j, ++n) {
                if (j == 0) {
                    for (int g = 0; g < NG && go; ++g) {
                        if (cnt[g] == 0)
                            continue;
                        go = wait(smem_u32(&sm.q_full[g]), (ph_q >> g) & 1);
                        ph_q ^= 1u << g;
                    }
                    go = go && wait(full(2 * n % kSt), (2 * n / kSt) & 1);
                    if (!go)
                        break;
                    tc_fence_after();
                    for (int g = 0; g < NG; ++g)
                        if (cnt[g] > 0)
                            qk(g, n);
                    if (elect_one())
                        tc_commit(empty(2 * n % kSt));
                    __syncwarp();
                }
                const uint32_t v_st = (2 * n + 1) % kSt;
                const uint32_t v_at = st_at + v_st * C::kTile;
                bool v_here = false, k_here = false;
                for (int g = 0; g < NG && go; ++g) {
                    if (j < cnt[g]) {
                        go = wait(smem_u32(&sm.p_full[g]), ph_p[g]);
                        ph_p[g] ^= 1;
                        if (go && !v_here) {
                            go = wait(full(v_st), ((2 * n + 1) / kSt) & 1);
                            v_here = true;
                        }
                        if (!go)
                            break;
                        tc_fence_after();
                        const int left = keys[g] - (s.kt0 + j) * kKeys;
                        const int steps = left >= kKeys ? kKeys / 16 : (left + 15) / 16;
                        if (elect_one()) {
                            for (int k = 0; k < steps; ++k)
                                mma_f16_ts(tmem + g * 256 + 128, tmem + g * 256 + k * 8,
                                           sdesc_sw128(v_at + k * 2 * kHalf * 1024, 1024, kHalf * 1024),
                                           Elem<T>::idesc(D, 1), (uint32_t)(j > 0 || k > 0));
                            if (j + 1 == cnt[g])
                                tc_commit(smem_u32(&sm.o_full[g]));
                        }
                        __syncwarp();
                    }
                    if (j + 1 < cnt[g]) {
                        if (!k_here) {
                            go = wait(full((2 * n + 2) % kSt), ((2 * n + 2) / kSt) & 1);
                            k_here = true;
                        }
                        if (!go)
                            break;
                        tc_fence_after();
                        qk(g, n + 1);
                    }
                }
                if (go && elect_one()) {
                    tc_commit(empty(v_st));
                    if (k_here)
                        tc_commit(empty((2 * n + 2) % kSt));
                }
                __syncwarp();
            }
        }
        if (*abort != 0) {
            // the MMAs in flight end (bounded) before their memory goes away
            if (elect_one()) {
                tc_commit(smem_u32(&sm.drain));
                mbar_wait_bounded(smem_u32(&sm.drain), 0, kTimeoutNs);
            }
            __syncwarp();
        }
    } else if (warp == C::kSoftmax + 2) {
        // ---- values at masked places
        uint32_t n = 0, seg = 0, ph_raw = 0;
        bool go = true;
        for (; go && walk.next(s); ++seg) {
            int all = group_keys<NG>(p, sm.len, s, NG - 1);
            if (NG == 2 && all == 0)
                all = group_keys<NG>(p, sm.len, s, 0);
            const int tiles = group_tiles(s, all);
            const int common = common_keys<NG>(p, sm.len, s);
            int32_t *const any = &sm.marks.any[seg % C::kMarks], *const from = sm.marks.from[seg % C::kMarks];
            bool clean = p.kv_len != nullptr;        // a decode step has no keys that only some rows see
            for (int j = 0; j < tiles && go; ++j, ++n) {
                const int k0 = (s.kt0 + j) * kKeys;
                if (k0 + kKeys <= common)
                    continue;
                if (!clean) {
                    for (int i = lane; i < D; i += 32)
                        from[i] = INT_MAX;
                    if (lane == 0)
                        *any = 0;
                    clean = true;
                    __syncwarp();
                }
                const uint32_t st = (2 * n + 1) % kSt;
                go = wait(smem_u32(&sm.raw[st]), (ph_raw >> st) & 1);
                ph_raw ^= 1u << st;
                if (!go)
                    break;
                uint8_t *const v = smem_raw + (NG + st) * C::kTile;
                // rows [common, all) are searched, rows behind them up to a step of the MMA zeroed
                const int lo = common > k0 ? common - k0 : 0;
                const int hi = all - k0 < kKeys ? all - k0 : kKeys;
                const int end = (hi + 15) / 16 * 16;
                // 16 bytes at a time: chunk x of row r is chunk x & 7 of half x >> 3, swizzled
                for (int i = lo * (D / 8) + lane; i < end * (D / 8); i += 32) {
                    const int r = i / (D / 8), x = i % (D / 8);
                    uint4 *const at = reinterpret_cast<uint4 *>(
                        v + ((r >> 3) * kHalf + (x >> 3)) * 1024 + (r & 7) * 128 +
                        (((x & 7) ^ (r & 7)) << 4));
                    if (r >= hi) {
                        *at = make_uint4(0, 0, 0, 0);
                        continue;
                    }
                    const uint4 y = *at;
                    if ((not_finite<T>(y.x) | not_finite<T>(y.y) | not_finite<T>(y.z) |
                         not_finite<T>(y.w)) == 0)
                        continue;
                    uint16_t *const e = reinterpret_cast<uint16_t *>(at);
                    for (int w = 0; w < 8; ++w)
                        if ((not_finite<T>(e[w]) & 0x8000u) != 0) {
                            atomicMin(&from[x * 8 + w], k0 + r);
                            e[w] = 0;
                            *any = 1;
                        }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(full(st));
            }
        }
    }
    } else {
        // ---- softmax: thread = row
        more_registers<C::kMoreRegs>();
        const int g = warp >> 2;
        const int r = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + g * 256 + lanes, o_at = s_at + 128;
        const uint32_t bar_q = smem_u32(&sm.q_full[g]), bar_s = smem_u32(&sm.s_full[g]);
        const uint32_t bar_p = smem_u32(&sm.p_full[g]), bar_o = smem_u32(&sm.o_full[g]);
        uint32_t ph_s = 0, ph_o = 0;
        // this thread's row of a segment: its token row, head and keys
        int64_t row = 0;
        int head = 0, keys = 0, gkeys = 0;
        bool ok = false;
        auto enter = [&](const Segment &x) {
            const int rr = (x.rt * NG + g) * 128 + r;
            ok = rr < x.rows;
            const int t = ok ? rr / p.group : 0;
            head = x.kvh * p.group + (ok ? rr - t * p.group : 0);
            gkeys = group_keys<NG>(p, sm.len, x, g);
            if (x.b < 0) {
                // prefix: the row of a request whose length is out of bounds is not written
                row = t;
                keys = p.prefix_len;
            } else if (p.kv_len != nullptr) {
                row = x.b;
                keys = sm.len[x.b];
            } else {
                row = (int64_t)p.row0[x.b] + t;
                keys = p.pos0[x.b] + t + 1;
            }
        };
        auto load_q = [&]() {
            const T *const src = static_cast<const T *>(p.q) + (ok ? row * p.q_stride + head * D : 0);
            const uint32_t dst = q_at + g * C::kTile + (uint32_t)r * 128;
#pragma unroll
            for (int c = 0; c < D / 8; ++c)
                cp_async_16(dst + (c >> 3) * 16384 + (((c & 7) ^ (r & 7)) << 4), src + c * 8, ok);
        };
        auto q_done = [&]() {
            cp_async_wait_all();
            fence_proxy_async_smem();
            mbar_arrive(bar_q);
        };
        bool have = walk.next(s), go = true;
        if (have) {
            enter(s);
            if (group_tiles(s, gkeys) > 0) {
                load_q();
                q_done();
            }
        }
        for (uint32_t seg = 0; have && go; ++seg) {
            const int tiles = group_tiles(s, gkeys);
            float m = -INFINITY, l = 0.f;       // m in units of log2, of scaled scores
            for (int j = 0; j < tiles; ++j) {
                go = wait(bar_s, ph_s);
                ph_s ^= 1;
                if (!go)
                    break;
                tc_fence_after();
                float x[kKeys];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    tmem_ld32(s_at + c * 32, *reinterpret_cast<float(*)[32]>(&x[c * 32]));
                tmem_wait_ld();
                const int valid = keys - (s.kt0 + j) * kKeys;
                if (__any_sync(0xffffffffu, valid < kKeys)) {
#pragma unroll
                    for (int c = 0; c < kKeys; ++c)
                        x[c] = c < valid ? x[c] : -INFINITY;
                }
                float t0 = x[0], t1 = x[1], t2 = x[2], t3 = x[3];
#pragma unroll
                for (int c = 4; c < kKeys; c += 4) {
                    t0 = fmaxf(t0, x[c]);
                    t1 = fmaxf(t1, x[c + 1]);
                    t2 = fmaxf(t2, x[c + 2]);
                    t3 = fmaxf(t3, x[c + 3]);
                }
                const float top = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3)) * p.scale_log2;
                const bool up = top > m + kLazy;
                if (__any_sync(0xffffffffu, up)) {
                    const float f = up ? ex2(m - top) : 1.f;
                    if (up)
                        m = top;
                    if (j > 0) {
                        // the previous product is done: the scores came after it
                        l *= f;
#pragma unroll
                        for (int c = 0; c < D; c += 32) {
                            float a[32];
                            tmem_ld32(o_at + c, a);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                a[i] *= f;
                            tmem_st32(o_at + c, a);
                        }
                    }
                }
                const float shift = m == -INFINITY ? 0.f : -m;
                float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
#pragma unroll
                for (int c = 0; c < kKeys; c += 32) {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float a0 = ex2(fmaf(x[c + 2 * i], p.scale_log2, shift));
                        const float a1 = ex2(fmaf(x[c + 2 * i + 1], p.scale_log2, shift));
                        const float a2 = ex2(fmaf(x[c + 2 * i + 2], p.scale_log2, shift));
                        const float a3 = ex2(fmaf(x[c + 2 * i + 3], p.scale_log2, shift));
                        l0 += a0;
                        l1 += a1;
                        l2 += a2;
                        l3 += a3;
                        w[i] = Elem<T>::pack(a0, a1);
                        w[i + 1] = Elem<T>::pack(a2, a3);
                    }
                    tmem_st16(s_at + c / 2, w);
                }
                l += (l0 + l1) + (l2 + l3);
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar_p);
            }
            if (!go)
                break;
            // the next segment's queries while the last product runs: the scores of this one's last
            // tile are here, so its queries are done with
            const Segment was = s;
            const int64_t was_row = row;
            const int was_head = head, was_keys = keys, was_tiles = tiles_of(gkeys);
            const bool was_ok = ok;
            have = walk.next(s);
            if (have) {
                enter(s);
                if (group_tiles(s, gkeys) > 0)
                    load_q();
            }
            if (tiles > 0) {
                go = wait(bar_o, ph_o);
                ph_o ^= 1;
                if (!go)
                    break;
                tc_fence_after();
            }
            if (have && group_tiles(s, gkeys) > 0)
                q_done();
            const bool marked = p.kv_len == nullptr && tiles > 0 &&
                                (was.kt1 < was_tiles ? was.kt1 : was_tiles) * kKeys >
                                    common_keys<NG>(p, sm.len, was) &&
                                *(volatile int32_t *)&sm.marks.any[seg % C::kMarks] != 0;
            const int32_t *const from = sm.marks.from[seg % C::kMarks];
            const bool direct = was.whole && p.prefix_len == 0;
            if (direct) {
                const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
                T *const o = static_cast<T *>(p.o) + was_row * p.o_stride + was_head * D;
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float a[32];
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
                            a[i] = was_keys > from[c + i] ? NAN : a[i];
                    }
                    if (was_ok) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4 *>(o + c + i) =
                                make_uint4(Elem<T>::pack(a[i] * inv, a[i + 1] * inv),
                                           Elem<T>::pack(a[i + 2] * inv, a[i + 3] * inv),
                                           Elem<T>::pack(a[i + 4] * inv, a[i + 5] * inv),
                                           Elem<T>::pack(a[i + 6] * inv, a[i + 7] * inv));
                    }
                }
                if (was_ok && p.lse != nullptr)
                    p.lse[was_row * p.n_heads + was_head] =
                        l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
            } else {
                int rows = 0;
                float *const slot = slot_of<D, NG>(p, was, cta, &rows);
                const int at = g * 128 + r;
                if (at < rows && was_ok)
                    reinterpret_cast<float2 *>(slot)[at] = make_float2(m, l);
                float *const a_at = slot + pairs_floats(rows) + (int64_t)at * D;
                if (tiles > 0) {
#pragma unroll
                    for (int c = 0; c < D; c += 32) {
                        float a[32];
                        tmem_ld32(o_at + c, a);
                        tmem_wait_ld();
                        if (marked) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                a[i] = was_keys > from[c + i] ? NAN : a[i];
                        }
                        if (at < rows && was_ok) {
#pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                *reinterpret_cast<float4 *>(a_at + c + i) =
                                    make_float4(a[i], a[i + 1], a[i + 2], a[i + 3]);
                        }
                    }
                }
            }
            tc_fence_before();
        }
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
// lse = ln 2 (M + log2 L).  A warp takes a row, D / 32 columns a lane; parts in the order of their
// keys, so that the same split gives the same bits.

template <int D>
struct Joined {
    float a[D / 32];
    float m = -INFINITY, l = 0.f;
    __device__ Joined()
    {
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
            a[i] = 0.f;
    }
    __device__ void add(const float *slot, int rows, int r, int lane)
    {
        const float2 ml = reinterpret_cast<const float2 *>(slot)[r];
        if (ml.x == -INFINITY && ml.y == 0.f)
            return;                                  // no key of this part: a is not written
        const float top = fmaxf(m, ml.x);
        const float f = ex2(m - top), h = ex2(ml.x - top);
        m = top;
        l = l * f + ml.y * h;
        const float *src = slot + pairs_floats(rows) + (int64_t)r * D + lane * (D / 32);
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
            a[i] = a[i] * f + src[i] * h;
    }
    template <typename T>
    __device__ void write(const AttnParams &p, int64_t row, int head, int lane) const
    {
        const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
        uint32_t *o = reinterpret_cast<uint32_t *>(static_cast<T *>(p.o) + row * p.o_stride + head * D +
                                                   lane * (D / 32));
#pragma unroll
        for (int i = 0; i < D / 32; i += 2)
            o[i / 2] = Elem<T>::pack(a[i] * inv, a[i + 1] * inv);
        if (p.lse != nullptr && lane == 0)
            p.lse[row * p.n_heads + head] = l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
    }
};

constexpr int kMergeWarps = 8;

// items split between CTAs: block (c, y) takes the item inside which CTA c's run begins, if it is the
// first one to begin there
template <typename T, int D, int NG>
__global__ void __launch_bounds__(kMergeWarps * 32)
attn_merge_kernel(const __grid_constant__ AttnParams p)
{
    __shared__ int32_t len[HS_MAX_BATCH];
    __shared__ Start start;
    __shared__ int own;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x + 1;
    if (warp == 0) {
        int before = 0;
        const int n = p.kv_len != nullptr ? read_lengths(p, len, lane, false, 0, &before) : 0;
        const Start st = find_start<NG>(p, len, n, c, lane);
        if (lane == 0) {
            start = st;
            own = n;
        }
    }
    __syncthreads();
    const Walk<NG> w(p, len, start);
    if (w.kt == 0 || w.u >= w.u1)
        return;
    const int64_t units = p.kv_len != nullptr ? (int64_t)own : p.units;
    const int64_t u0 = w.u - w.kt, u1 = u0 + w.tiles();    // the item's units
    const int c0 = cta_of(units, p.ctas, u0), c1 = cta_of(units, p.ctas, u1 - 1);
    if (c0 != cta_of(units, p.ctas, w.u - 1))
        return;
    const int rows = slot_rows<NG>(p);
    const int64_t size = slot_floats<D>(rows);
    const int all = w.rows();
    for (int r = blockIdx.y * kMergeWarps + warp; r < rows; r += gridDim.y * kMergeWarps) {
        const int rr = w.rt * 128 * NG + r;
        if (rr >= all)
            break;
        Joined<D> x;
        x.add(p.part + (2 * c0 + 1) * size, rows, r, lane);
        for (int i = c; i <= c1; ++i)
            if (has_units(units, p.ctas, i))
                x.add(p.part + 2 * i * size, rows, r, lane);
        const int t = rr / p.group;
        x.template write<T>(p, p.kv_len != nullptr ? w.b : (int64_t)p.row0[w.b] + t,
                            w.kvh * p.group + rr - t * p.group, lane);
    }
}

// behind a shared prefix: block (request, KV head), a warp per head
template <typename T, int D, int NG>
__global__ void __launch_bounds__(kMergeWarps * 32)
attn_merge_shared_kernel(const __grid_constant__ AttnParams p)
{
    __shared__ int32_t len[HS_MAX_BATCH];
    __shared__ int sums[2];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = blockIdx.x / p.n_kv, kvh = blockIdx.x - b * p.n_kv;
    if (warp == 0) {
        int before = 0;
        const int n = read_lengths(p, len, lane, false, b, &before);
        if (lane == 0) {
            sums[0] = before;
            sums[1] = n;
        }
    }
    __syncthreads();
    if (len[b] < 0)
        return;
    const int per = tiles_of(p.prefix_len), own = len[b] > 0 ? tiles_of(len[b]) : 1;
    const int64_t pre = (int64_t)per * p.n_kv * row_tiles<NG>(p.batch * p.group);
    const int64_t units = pre + sums[1];
    const int64_t u0 = pre + sums[0] + (int64_t)kvh * own;
    const int item = b * p.n_kv + kvh;
    // an unsplit item belongs to the CTA in whose run it begins
    const int c0 = cta_of(units, p.ctas, u0);
    const int c1 = p.unsplit ? c0 : cta_of(units, p.ctas, u0 + own - 1);
    const float *const own_at = p.part + prefix_part_floats<D, NG>(p);
    for (int h = warp; h < p.group; h += kMergeWarps) {
        const int rr = b * p.group + h, rt = rr / (128 * NG), r = rr - rt * 128 * NG;
        const int pitem = rt * p.n_kv + kvh;
        const int p0 = cta_of(units, p.ctas, (int64_t)pitem * per);
        const int p1 = p.unsplit ? p0 : cta_of(units, p.ctas, (int64_t)(pitem + 1) * per - 1);
        Joined<D> x;
        for (int c = p0; c <= p1; ++c)
            if (has_units(units, p.ctas, c))
                x.add(p.part + (pitem + c) * slot_floats<D>(128 * NG), 128 * NG, r, lane);
        for (int c = c0; c <= c1; ++c)
            if (has_units(units, p.ctas, c))
                x.add(own_at + (item + c) * slot_floats<D>(p.group), p.group, h, lane);
        x.template write<T>(p, b, kvh * p.group + h, lane);
    }
}

// ---- launches ------------------------------------------------------------------------------

PFN_cuTensorMapEncodeTiled_v12000 encode_fn()
{
    // resolved once per process from the driver; a pure function pointer
    static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> fn{nullptr};
    PFN_cuTensorMapEncodeTiled_v12000 f = fn.load(std::memory_order_acquire);
    if (f == nullptr) {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault,
                                             &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess) {
            f = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
            fn.store(f, std::memory_order_release);
        }
    }
    return f;
}

// The cache of a layer as [8-token group][64-element block of a token's heads][token][64]: a copy's
// box is one head of a page (or of 128 keys of one), 8-token groups outermost, which in shared
// memory is the operand layout of both products: 128-byte rows, swizzled, in atoms of 8 tokens, the
// atoms of a row's blocks side by side.
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
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int prefill_rows(const AttnParams &p)
{
    int most = 0;
    for (int b = 0; b < p.batch; ++b)
        most = p.n_tokens[b] > most ? p.n_tokens[b] : most;
    return most * p.group;
}

// tiles of rows of an item: two where a request (or the rows in front of a shared prefix) has them
int groups_of(const AttnParams &p)
{
    if (p.kv_len == nullptr)
        return prefill_rows(p) > 128 ? 2 : 1;
    return p.prefix_len > 0 && p.batch * p.group > 128 ? 2 : 1;
}

template <int NG>
void plan_prefill(AttnParams &p, int most)
{
    int64_t units = 0;
    for (int b = 0; b < p.batch; ++b)
        for (int rt = 0; rt < row_tiles<NG>(p.n_tokens[b] * p.group); ++rt)
            units += (int64_t)p.n_kv * prefill_tiles<NG>(p.pos0[b], p.n_tokens[b], p.group, rt);
    p.units = units;
    p.ctas = (int)(units < most ? units : most);
    int c = 0;
    int64_t u = 0;
    for (int b = 0; b < p.batch && c < p.ctas; ++b)
        for (int rt = 0; rt < row_tiles<NG>(p.n_tokens[b] * p.group) && c < p.ctas; ++rt) {
            const int n = prefill_tiles<NG>(p.pos0[b], p.n_tokens[b], p.group, rt);
            for (; c < p.ctas && first_unit(units, p.ctas, c) < u + (int64_t)n * p.n_kv; ++c) {
                const int64_t v = first_unit(units, p.ctas, c) - u;
                p.start_b[c] = (int16_t)b;
                p.start_item[c] = rt * p.n_kv + (int)(v / n);
                p.start_kt[c] = (int)(v % n);
            }
            u += (int64_t)n * p.n_kv;
        }
}

template <typename T, int D, int NG>
cudaError_t launch(const AttnParams &p, cudaStream_t s)
{
    CUtensorMap map;
    if (!encode_cache<D>(&map, p))
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> smem_set{0};
    cudaError_t e = launch_pdl_big_smem(attn_kernel<T, D, NG>, dim3((unsigned)p.ctas),
                                        dim3(Cfg<D, NG>::kThreads), smem_bytes<D, NG>(), s, smem_set, p,
                                        map);
    if (e != cudaSuccess)
        return e;
    if (p.prefix_len > 0)
        return launch_pdl(attn_merge_shared_kernel<T, D, NG>, dim3((unsigned)(p.batch * p.n_kv)),
                          dim3(kMergeWarps * 32), 0, s, p);
    if (p.unsplit || p.ctas == 1)
        return cudaSuccess;
    const int rows = slot_rows<NG>(p);
    const int blocks = (rows + kMergeWarps - 1) / kMergeWarps;
    return launch_pdl(attn_merge_kernel<T, D, NG>, dim3((unsigned)(p.ctas - 1), (unsigned)(blocks < 8 ? blocks : 8)),
                      dim3(kMergeWarps * 32), 0, s, p);
}

template <typename T>
cudaError_t launch(const AttnParams &p, int d, cudaStream_t s)
{
    if (groups_of(p) == 2)
        return d == 128 ? launch<T, 128, 2>(p, s) : launch<T, 64, 2>(p, s);
    return d == 128 ? launch<T, 128, 1>(p, s) : launch<T, 64, 1>(p, s);
}

}  // namespace

int64_t plan_attn(AttnParams &p, int d, int sm_count)
{
    const int ng = groups_of(p);
    int most = sm_count * (ng == 2 ? 1 : 2);
    if (most > kAttnMaxCtas)
        most = kAttnMaxCtas;
    auto slot = [&](int rows) {
        return (int64_t)sizeof(float) * (d == 128 ? slot_floats<128>(rows) : slot_floats<64>(rows));
    };
    if (p.kv_len == nullptr) {
        if (ng == 2)
            plan_prefill<2>(p, most);
        else
            plan_prefill<1>(p, most);
        return p.unsplit || p.ctas == 1 ? 0 : 2 * p.ctas * slot(128 * ng);
    }
    const int64_t own = (int64_t)p.batch * p.n_kv * (p.max_kv > 0 ? tiles_of(p.max_kv) : 1);
    const int64_t items = (ng == 2 ? row_tiles<2>(p.batch * p.group) : row_tiles<1>(p.batch * p.group)) *
                          (int64_t)p.n_kv;
    const int64_t units = own + items * tiles_of(p.prefix_len);
    p.ctas = (int)(units < most ? units : most);
    if (p.prefix_len > 0)
        return (items + p.ctas) * slot(128 * ng) + ((int64_t)p.batch * p.n_kv + p.ctas) * slot(p.group);
    return p.unsplit || p.ctas == 1 ? 0 : 2 * p.ctas * slot(p.group);
}

cudaError_t launch_attn(const AttnParams &p, int d, int dtype, cudaStream_t s)
{
    return dtype == HS_FP16 ? launch<__half>(p, d, s) : launch<__nv_bfloat16>(p, d, s);
}

}  // namespace hs
