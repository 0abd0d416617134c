// The walk of the attention kernels (attn_tc.cuh) over a call's work: units, items, segments, and where
// partial results lie.
#pragma once

#include <climits>

#include "attn_internal.cuh"

namespace hs {
namespace attn {

constexpr int kKeys = 128;               // keys per tile

// where a CTA's run of units begins and ends
struct Start {
    int32_t u, left;                     // its first unit and how many
    int32_t b, rt, kvh, at;
};

// ---- the walk over items -------------------------------------------------------------------

__host__ __device__ __forceinline__ int tiles_of(int keys)
{
    return (keys + kKeys - 1) / kKeys;
}

// the first unit of CTA c's run (c <= 320; small numbers without the slow division)
__host__ __device__ __forceinline__ int first_unit(int units, int ctas, int c)
{
    if (units < 1 << 22)
        return (int)((uint32_t)units * (uint32_t)c / (uint32_t)ctas);
    return (int)((int64_t)units * c / ctas);
}

// the CTA that has unit u: the largest c with first_unit(c) <= u
__host__ __device__ __forceinline__ int cta_of(int units, int ctas, int u)
{
    if (units < 1 << 22)
        return (int)(((uint32_t)(u + 1) * (uint32_t)ctas - 1) / (uint32_t)units);
    return (int)((((int64_t)u + 1) * ctas - 1) / units);
}

__device__ __forceinline__ bool has_units(int units, int ctas, int c)
{
    return first_unit(units, ctas, c) < first_unit(units, ctas, c + 1);
}

// b = -1 stands for the shared prefix, whose rows are those of all requests
template <int NG>
__host__ __device__ __forceinline__ int row_tiles(int rows)
{
    return (rows + 128 * NG - 1) / (128 * NG);
}

// prefill: keys of the last row before row `end` of a request
__device__ __forceinline__ int keys_before(const AttnParams &p, int pos0, int end)
{
    return pos0 + p.by_group.div(end - 1) + 1;
}

// prefill: key tiles of a request's row tile
template <int NG>
int prefill_tiles(int pos0, int n_tokens, int group, int rt)
{
    const int rows = n_tokens * group, end = (rt + 1) * 128 * NG;
    return tiles_of(pos0 + ((end < rows ? end : rows) - 1) / group + 1);
}

// Whether a call of `units` units is better not split: a join costs what 3 tiles cost (2 to 4 us), and a
// second launch its host time; whole items leave a CTA at most the longest above an even share (with an item
// or less to each, the longest).  One request of 2 heads with 256 keys: 6.2 us a call, host bound, instead of
// 9 split.
inline bool better_whole(const AttnParams &p, int64_t items, int longest, int64_t units)
{
    const int64_t even = units / p.ctas - p.extra, share = even > 1 ? even : 1;
    return (items <= p.ctas ? 0 : share) + longest <= share + 3;
}

// How long a wait may take.  Most are for a step of one tile (3 us at most, with HBM shared by all), but the
// warps that search values, and a group of rows without any in a segment, wait for another one's whole run of
// tiles: the longest item and an even share at most.  (At 0.65 us a tile one CTA's 200 million keys
// take longer than 1 s.)
inline uint64_t wait_limit_ns(const AttnParams &p, int longest, int64_t units)
{
    return 1000000000ull + 20000ull * (uint64_t)(units / p.ctas + longest);
}

// one item's key tiles [kt0, kt1) as one CTA has them
struct Segment {
    int b, rt, kvh, kt0, kt1;
    int rows;        // of the whole request (or of all, for the prefix)
    bool whole;      // all of the item's key tiles
    int item;        // running number of the item within its part (prefix or requests), decode only
};

template <int NG, class Plan>
struct Walk {
    const AttnParams &p;
    const Plan &plan;
    const int32_t *len;                  // decode: the lengths in shared memory
    int left;                            // units of the run not yet given out
    int b, rt, kvh, at;                  // the item at hand and its units given out

    __device__ int rows() const
    {
        if (b < 0)
            return p.batch * p.group;
        if constexpr (Plan::kDecode)
            return p.group;
        else
            return plan.req[b].n * p.group;
    }
    __device__ int tiles() const
    {
        if (b < 0)
            return tiles_of(p.prefix_len);
        if constexpr (Plan::kDecode)
            return len[b] > 0 ? tiles_of(len[b]) : 1;   // an empty row is written by someone
        else
            return tiles_of(keys_before(p, plan.req[b].pos0, min(rows(), (rt + 1) * 128 * NG)));
    }
    __device__ int extra() const
    {
        return b < 0 ? p.extra_shared : p.extra;
    }
    __device__ bool skip() const
    {
        if constexpr (Plan::kDecode)
            return len[b] < 0;
        else
            return plan.req[b].n == 0;
    }
    __device__ void next_item()
    {
        at = 0;
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
    __device__ Walk(const AttnParams &params, const Plan &plan_, const int32_t *lens, const Start &s)
        : p(params), plan(plan_), len(lens), left(s.left), b(s.b), rt(s.rt), kvh(s.kvh), at(s.at)
    {
        if (p.unsplit && left > 0 && at != 0) {       // begins with the next whole item
            left -= tiles() + extra() - at;
            next_item();
        }
    }
    __device__ bool next(Segment &s)
    {
        while (left > 0) {
            const int n = tiles(), extra = this->extra();
            int end = n + extra;
            if (!p.unsplit && end - at > left)
                end = at + left;
            s.kt0 = at > extra ? at - extra : 0;
            s.kt1 = end > extra ? end - extra : 0;
            s.b = b;
            s.rt = rt;
            s.kvh = kvh;
            s.rows = rows();
            s.whole = s.kt1 - s.kt0 == n;
            s.item = (b < 0 ? rt : b) * p.n_kv + kvh;
            left -= end - at;
            at = end;
            if (at == n + extra)
                next_item();
            if (s.kt1 > s.kt0)
                return true;
        }
        return false;
    }
    // keys that the last row of group g of a segment's row tile attends to (0: the group has no row)
    __device__ int group_keys(const Segment &s, int g) const
    {
        const int r0 = (s.rt * NG + g) * 128;
        if (r0 >= s.rows)
            return 0;
        if (s.b < 0)
            return p.prefix_len;
        if constexpr (Plan::kDecode)
            return len[s.b];
        else
            return keys_before(p, plan.req[s.b].pos0, min(s.rows, r0 + 128));
    }
    // the same of its last group that has rows
    __device__ int all_keys(const Segment &s) const
    {
        const int n = group_keys(s, NG - 1);
        return NG == 2 && n == 0 ? group_keys(s, 0) : n;
    }
    // keys that every row of the segment's item attends to
    __device__ int common_keys(const Segment &s) const
    {
        if (s.b < 0)
            return p.prefix_len;
        if constexpr (Plan::kDecode)
            return len[s.b];
        else
            return keys_before(p, plan.req[s.b].pos0, s.rt * 128 * NG + 1);
    }
};

// tiles of the segment that a group with `keys` keys takes part in
__device__ __forceinline__ int group_tiles(const Segment &s, int keys)
{
    const int n = tiles_of(keys);
    const int end = n < s.kt1 ? n : s.kt1;
    return end > s.kt0 ? end - s.kt0 : 0;
}

// decode: units of an item of `len` keys, and of a request (0: its length is out of bounds)
__device__ __forceinline__ int item_units(const AttnParams &p, int len)
{
    return (len > 0 ? tiles_of(len) : 1) + p.extra;
}

__device__ __forceinline__ int own_units(const AttnParams &p, int len)
{
    return len < 0 ? 0 : item_units(p, len) * p.n_kv;
}

// units of an item of the shared prefix (0: there is none)
__host__ __device__ __forceinline__ int prefix_units(const AttnParams &p)
{
    return p.prefix_len > 0 ? tiles_of(p.prefix_len) + p.extra_shared : 0;
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
    constexpr int kAhead = 6;             // loads that do not wait for one another; HS_MAX_BATCH takes two rounds
    int sum = 0, part = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32 * kAhead) {
        int n[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int b = b0 + i * 32 + lane;
            n[i] = b < p.batch ? p.kv_len[b] : -1;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int b = b0 + i * 32 + lane;
            if (b < p.batch) {
                if (n[i] < 0 || n[i] > p.max_kv) {
                    if (complain)
                        report(p.d_err, HS_DEVERR_LENGTH);
                    n[i] = -1;
                }
                len[b] = n[i];
            }
            const int x = own_units(p, n[i]);
            sum += x;
            part += b < upto ? x : 0;
        }
    }
    __syncwarp();
    *before = __reduce_add_sync(0xffffffffu, part);
    return __reduce_add_sync(0xffffffffu, sum);
}

// where CTA c's run begins
template <int NG>
__device__ __forceinline__ Start find_start(const AttnParams &p, const PrefillPlan &plan, int c)
{
    Start s;
    s.u = first_unit(p.units, p.ctas, c);
    s.left = first_unit(p.units, p.ctas, c + 1) - s.u;
    const PrefillPlan::Cta at = plan.cta[c];
    s.b = at.b;
    s.rt = p.by_kv.div(at.item);
    s.kvh = at.item - s.rt * p.n_kv;
    s.at = at.unit;
    return s;
}

// the same of a decode step (one warp; the lengths in shared memory, `own` their units)
template <int NG>
__device__ __forceinline__ Start find_start(const AttnParams &p, const int32_t *len, int own, int c,
                                            int lane)
{
    Start s;
    const int per = prefix_units(p);
    const int pre = per * p.n_kv * row_tiles<NG>(p.batch * p.group);
    const int units = pre + own;
    s.u = first_unit(units, p.ctas, c);
    s.left = first_unit(units, p.ctas, c + 1) - s.u;
    s.b = -1;
    s.rt = s.kvh = s.at = 0;
    if (s.u < pre) {
        const int item = s.u / per;
        s.at = s.u - item * per;
        s.rt = item / p.n_kv;
        s.kvh = item - s.rt * p.n_kv;
        return s;
    }
    int v = s.u - pre;                 // the request with unit v of all requests'
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const int b = b0 + lane;
        const int x = own_units(p, b < p.batch ? len[b] : -1);
        const int incl = warp_scan(x, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, v < incl);
        const int last = __shfl_sync(0xffffffffu, incl, 31);
        if (hit != 0) {
            const int first = __ffs(hit) - 1;
            v -= __shfl_sync(0xffffffffu, incl - x, first);
            s.b = b0 + first;
            const int n = item_units(p, len[s.b]);
            s.kvh = v / n;
            s.at = v - s.kvh * n;
            return s;
        }
        v -= last;
    }
    return s;                                 // no unit is left
}

// ---- partial results -----------------------------------------------------------------------
//
// A slot holds R rows: R pairs (m, l), padded to 16 bytes, then the sums a: of decode R rows of D
// floats, of prefill D columns of R (a warp stores 32 rows of a column, and the join reads them so).
// Without a shared prefix an item leaves a partial result in at most two places of a CTA's run: at its
// beginning, where it does not start the item (slot 2 cta), and at its end, where it does (slot
// 2 cta + 1).  Behind a shared prefix every segment is partial; its slot is item + cta, which no other
// segment of its part (prefix, requests) has, since both only grow along the run.

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

// where a segment's slot lies in the workspace, in floats
template <int D, int NG, class Plan>
__device__ __forceinline__ int64_t slot_of(const AttnParams &p, const Segment &s, int cta, int *rows)
{
    if (s.b < 0) {
        *rows = 128 * NG;
        return (int64_t)(s.item + cta) * slot_floats<D>(128 * NG);
    }
    *rows = Plan::kDecode ? p.group : 128 * NG;
    if (Plan::kDecode && p.prefix_len > 0)
        return prefix_part_floats<D, NG>(p) + (int64_t)(s.item + cta) * slot_floats<D>(*rows);
    return (int64_t)(2 * cta + (s.kt0 == 0)) * slot_floats<D>(*rows);
}

}  // namespace attn
}  // namespace hs
