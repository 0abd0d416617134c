// New tokens' K and V rows of one layer quantised into their 8-bit pages, alone or with rotary positions on
// the way (the FP8 KV setting, Table 1 of the paper).
//
// Of a group of 16 tokens, KV head and plane: M = max |x| of the new values, need = the smallest
// 2^e >= M / 448, scale = need (a group that begins) or max(scale, need) (one that goes on; where it grows, the
// bytes that the group holds are rounded to the new scale), bytes = E4M3(x / scale).  With powers of two
// both divisions are exact, so each value is rounded once for each scale that it lives under.
//
// The rows of a group stand one behind the other, but for skipped ones: its first row's place (the last row in front that is
// not skipped has another group) says who owns it.  Values and keys that are not turned are taken by warps, a (KV head, plane) of a group at a time with its
// 16 rows in registers, so that M and the bytes come from one read.  Keys that are turned are taken by teams of D threads, a
// lane 16 values of one row, and q by blocks of their own, as hs_rope_apply does.
//
// Bound by HBM where there are many rows: 28,913 rows of 8 x 128 keys and values (178 MB) take 29.5 us, 6.0 TB/s; with
// positions and 32 heads of q, 28,000 rows 107 us, 6.0 TB/s; 14,494 rows of 16 + 4 heads 30.6 us, 5.3.  A step of 64 rows
// with positions takes 4.2 us: four loads that wait for one another, sines and cosines, a meeting of four warps a head.
//
// Turned values are good to 2^-21 of |x| + |y|: the angle is good to 2^-25 half turns, sines and cosines to 2^-24, and four
// more roundings follow (sum 2^-21.3), which leaves room for 2^-23.3 radians that the 64 bits of an angle lack at
// positions up to 2^39.  What lies nearer than that to a border, of two scales or of two E4M3 numbers, is
// decided by its value in twice as many bits (of an angle: 96), so that the bytes are those of the exactly turned keys.
#include "attn_ptx.cuh"
#include "kv8_internal.cuh"

namespace hs {
namespace {

using namespace kv8;

constexpr int kThreads = 128;
constexpr float kOff = 0x1p-21f;

// The upper half of a product of 64 bits, to 2 units: what the lower halves carry is left out.
__device__ __forceinline__ uint64_t upper(uint64_t a, uint64_t b)
{
    const uint32_t ah = a >> 32, bh = b >> 32;
    return (uint64_t)ah * bh + __umulhi(ah, (uint32_t)b) + __umulhi((uint32_t)a, bh);
}

// A number as high + low, to 2^-47 of it.
struct Two {
    float high, low;
};

// magnitude 2^-63, with a sign
__device__ __forceinline__ Two two_of(uint64_t magnitude, bool negative)
{
    const float sign = negative ? -1.f : 1.f;
    return {(float)(uint32_t)(magnitude >> 39) * (0x1p-24f * sign),
            (float)((uint32_t)(magnitude >> 15) & 0xffffffu) * (0x1p-48f * sign)};
}

// Element `second` of the pair (x, y) times `by` turned, to 2^-45 of |x| + |y|: what lies next to a border of rounding is
// decided by it.  The angle's sine and cosine are Taylor's series of at most an eighth of a turn in integers of 64 bits
// (to 2^-54), which need neither tables nor the float64 units: with those a step of 64 rows took 1 us more.
__device__ __noinline__ Two turned_closely(int64_t angle, Two gain, float x, float y, float by, bool second)
{
    // angle = quarter 2^62 + r, -2^61 <= r <= 2^61
    const uint64_t a = (uint64_t)angle, quarter = (a + (1ull << 61)) >> 62, r = a - (quarter << 62);
    const bool below = (int64_t)r < 0;
    // of 2^64: the angle in radians, and its square
    const uint64_t t = 2 * upper((below ? -r : r) << 2, 0xc90fdaa22168c235ull), u = upper(t, t);
    uint64_t s = 0xd73f9f, c = 0xd73fa;                // 1 / 15!, 1 / 16!
    s = 0xb092309dull - upper(u, s);                   // 1 / 13!
    c = 0xc9cba54ull - upper(u, c);                    // 1 / 14!
    s = 0x6b99159fd5ull - upper(u, s);                 // and so on
    c = 0x8f76c77fcull - upper(u, c);
    s = 0x2e3bc74aad8eull - upper(u, s);
    c = 0x49f93edde28ull - upper(u, c);
    s = 0xd00d00d00d00dull - upper(u, s);
    c = 0x1a01a01a01a02ull - upper(u, c);
    s = 0x222222222222222ull - upper(u, s);
    c = 0x5b05b05b05b05bull - upper(u, c);
    s = 0x2aaaaaaaaaaaaaabull - upper(u, s);
    c = 0xaaaaaaaaaaaaaabull - upper(u, c);
    c = 0x8000000000000000ull - upper(u, c);
    s = (t - upper(t, upper(u, s))) >> 1;              // of 2^63
    c = (1ull << 63) - (upper(u, c) >> 1);
    // cos, sin of quarters 0 to 3: (c, s), (-s, c), (-c, -s), (s, -c)
    const bool odd = quarter & 1, high = quarter & 2;
    const Two cosine = two_of(odd ? s : c, odd ? below == high : high),
              sine = two_of(odd ? c : s, odd ? high : below != high);
    // p cos + q sin, the products' and the sum's errors added behind
    const float p = by * (second ? y : x), q = by * (second ? x : -y);
    const float f = p * cosine.high, g = q * sine.high, h = f + g, k = h - f;
    const float l = ((f - (h - k)) + (g - k)) + (fmaf(p, cosine.high, -f) + fmaf(q, sine.high, -g)) +
                    (p * cosine.low + q * sine.low);
    const float m = h * gain.high, n = fmaf(h, gain.high, -m) + (h * gain.low + l * gain.high);
    const float sum = n == 0.f ? m : m + n;            // a zero keeps its sign
    return {sum, n - (sum - m)};
}

// a float that E4M3 rounds to the same number as x: nearest, but never onto a midpoint that it is not
__device__ __forceinline__ float toward(Two x)
{
    const uint32_t bits = __float_as_uint(x.high);
    if ((bits & 0x7ffff) == 0 && x.low != 0.f)
        return __uint_as_float(bits + ((x.low > 0.f) == (x.high > 0.f) ? 1 : -1));
    return x.high;
}

// 448 2^e is 1.75 2^(e + 8): the e of the smallest 2^e >= x / 448, for the bits of a float x > 0
__device__ __forceinline__ int exponent_of(uint32_t bits)
{
    return (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
}

// eight pairs as the bytes of a lane's vectors: words 0 and 1 of the first, 2 and 3 of the second
template <bool kHalf>
__device__ __forceinline__ void bytes_of(const Pairs &p, uint32_t (&w)[4])
{
    float2 x[4], y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[k] = ptx::unpair(p.x[k]);
        y[k] = ptx::unpair(p.y[k]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (kHalf) {
            w[i] = to_e4m3(x[2 * i].x, x[2 * i].y, x[2 * i + 1].x, x[2 * i + 1].y);
            w[i + 2] = to_e4m3(y[2 * i].x, y[2 * i].y, y[2 * i + 1].x, y[2 * i + 1].y);
        } else {
            w[2 * i] = to_e4m3(x[2 * i].x, y[2 * i].x, x[2 * i].y, y[2 * i].y);
            w[2 * i + 1] = to_e4m3(x[2 * i + 1].x, y[2 * i + 1].x, x[2 * i + 1].y, y[2 * i + 1].y);
        }
    }
}

// what a warp needs of the group whose rows it quantises
struct Group {
    uint8_t *at;                  // its first token's bytes of the KV head's plane
    float *scale_at;
    float old;
    unsigned tokens;              // that get rows
    unsigned rows;                // of the 16 from the first one on
    int spot;                     // lane i: the token of row i
};

// Settles the group's scale, rounds what it holds to it where it grows, and gives the scale.
template <int D>
__device__ __forceinline__ float settle(const Group &g, int e, int lane)
{
    constexpr int kLanes = D / 16, kAtOnce = 32 / kLanes;
    const float need = power_of_two(e < -126 ? -126 : e);
    const bool anew = g.tokens & 1;
    const float scale = anew ? need : fmaxf(g.old, need);
    if (!anew && need > g.old) {
        // 16 bytes to a lane
        const float shrink = g.old / need;
#pragma unroll 1
        for (int i = lane / kLanes; i < kGroup; i += kAtOnce) {
            if ((g.tokens >> i) & 1)
                continue;
            uint4 *const w = reinterpret_cast<uint4 *>(g.at + i * D) + lane % kLanes;
            const uint4 y = *w;
            auto again = [&](uint32_t u) {
                const float2 f = widen<__half>(e4m3_to_f16(u)), h = widen<__half>(e4m3_to_f16_high(u));
                return to_e4m3(f.x * shrink, f.y * shrink, h.x * shrink, h.y * shrink);
            };
            *w = make_uint4(again(y.x), again(y.y), again(y.z), again(y.w));
        }
    }
    if (lane == 0)
        *g.scale_at = scale;
    return scale;
}

// Rows of values that are quantised as they are: row i of the group at from + i * stride.
template <typename T, int D>
__device__ __forceinline__ void quantise(const Group &g, const uint4 *from, int64_t stride, int lane)
{
    constexpr int kLanes = D / 16, kAtOnce = 32 / kLanes, kSteps = kGroup / kAtOnce;
    constexpr uint32_t kInf = std::is_same<T, __half>::value ? 0x7c00 : 0x7f80;
    const int v = lane % kLanes, sub = lane / kLanes;
    const unsigned on = g.rows >> sub;
    uint4 in[kSteps][2];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int i = s * kAtOnce + sub;
        in[s][0] = in[s][1] = make_uint4(0, 0, 0, 0);
        if (on & (1u << s * kAtOnce)) {
            in[s][0] = __ldcs(from + i * stride + v);
            in[s][1] = __ldcs(from + i * stride + v + kLanes);
        }
    }
    // the largest of the magnitudes' bits
    uint32_t top = 0;
    auto most = [&](uint32_t x) { asm("max.u16x2 %0, %0, %1;" : "+r"(top) : "r"(x & 0x7fff7fffu)); };
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            most(in[s][h].x), most(in[s][h].y), most(in[s][h].z), most(in[s][h].w);
        }
    top = __reduce_max_sync(0xffffffffu, max(top & 0xffff, top >> 16));
    const bool odd = top >= kInf;                      // a value that is not finite
    if (odd) {
        top = 0;
        auto finite = [&](uint32_t x) { top = (x & 0x7fff) < kInf ? max(top, x & 0x7fff) : top; };
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t u[4] = {in[s][h].x, in[s][h].y, in[s][h].z, in[s][h].w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    finite(u[j]), finite(u[j] >> 16);
            }
        top = __reduce_max_sync(0xffffffffu, top);
    }
    const float by = inverse(settle<D>(g, exponent_of(__float_as_uint(widen<T>(top).x)), lane));
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int i = s * kAtOnce + sub, token = __shfl_sync(0xffffffffu, g.spot, i);
        if (!(on & (1u << s * kAtOnce)))
            continue;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t u[4] = {in[s][h].x, in[s][h].y, in[s][h].z, in[s][h].w};
            uint32_t y[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float2 a = widen<T>(u[2 * j]), b = widen<T>(u[2 * j + 1]);
                if (odd) {                             // an infinity becomes NaN
                    a.x += 0.f * a.x, a.y += 0.f * a.y;
                    b.x += 0.f * b.x, b.y += 0.f * b.y;
                }
                y[j] = to_e4m3(a.x * by, a.y * by, b.x * by, b.y * by);
            }
            *reinterpret_cast<uint2 *>(g.at + token * D + 8 * (v + h * kLanes)) = make_uint2(y[0], y[1]);
        }
    }
}

// The groups that begin in a window of 16 rows: lane l of each warp has the slot of row `first` + l, -1 if it is skipped.
// A group's rows lie within 16, with none but skipped ones among them, so that 32 rows in front say whether one begins it.
// `meanwhile` is done while the slots are on their way, given the row behind `first`.
struct Window {
    int64_t first, slot;
    unsigned begins;              // lanes whose row begins a group
    template <typename F>
    __device__ __forceinline__ Window(const Kv8Append &p, int64_t row, bool complain, int lane, F meanwhile) : first(row - 1)
    {
        const int64_t mine = first + lane;
        slot = -1;
        if (mine >= 0 && mine < p.n_rows)
            asm volatile("ld.global.nc.b64 %0, [%1];" : "=l"(slot) : "l"(p.slots + mine));
        meanwhile(row);
        if (slot >= p.cache.num_blocks << p.cache.page_shift) {
            if (complain && lane > 0 && lane <= kGroup)
                report(p.d_err, HS_DEVERR_BLOCK_OOB);
            slot = -1;
        }
        slot = slot < 0 ? -1 : slot;
        // the group of the last row in front that is not skipped
        const unsigned taken = __ballot_sync(0xffffffffu, slot >= 0), front = taken & ((1u << lane) - 1);
        int64_t before = __shfl_sync(0xffffffffu, group(), front != 0 ? 31 - __clz(front) : 0);
        if (!(taken & 1) && first > 0) {
            int64_t older = -1;
            if (mine >= 32)
                older = __ldg(p.slots + (mine - 32));
            older = older >= p.cache.num_blocks << p.cache.page_shift ? -1 : older;
            const unsigned some = __ballot_sync(0xffffffffu, older >= 0);
            older = __shfl_sync(0xffffffffu, older, some != 0 ? 31 - __clz(some) : 0);
            if (front == 0)
                before = some != 0 ? older >> 4 : -1;
        }
        begins = __ballot_sync(0xffffffffu, lane >= 1 && lane <= kGroup && slot >= 0 && group() != before);
    }
    __device__ __forceinline__ int64_t group() const { return slot >> 4; }
    // which of the 16 rows from lane l's on are of its group
    __device__ __forceinline__ unsigned rows(int l) const
    {
        return __ballot_sync(0xffffffffu, group() == __shfl_sync(0xffffffffu, group(), l)) >> l & 0xffffu;
    }
};

// Brings a head's 16 rows from row `first` on to L2 while the slots that say whose they are come: 28,913 rows of 8 x 128 29.5
// us, 31.4 without; 4,000 of 32 + 8 x 128 with positions 18.7, 19.9.
template <int D>
__device__ __forceinline__ void ahead(const Kv8Append &p, const uint4 *head, int64_t first, int lane)
{
    constexpr int kLines = D / 64;                     // of 128 bytes to a row
#pragma unroll
    for (int i = lane / kLines; i < kGroup; i += 32 / kLines)
        if (first + i < p.n_rows)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(head + (first + i) * p.kv_stride + lane % kLines * 8));
}

// Who shares a window takes a run of its (group, plane) pairs, the planes of a group one after the other: of a prompt's window
// one group's, of a step's up to 16 groups'.  f(lane whose row begins the group, its planes `from` up to `to`).  Windows of
// fewer rows, of which most begin nothing in a prompt, took 15 % longer for 1,000 rows of 8 x 128.
template <typename F>
__device__ __forceinline__ void share(unsigned begins, int planes, int part, int parts_log, F f)
{
    const int all = __popc(begins) * planes;
    int from = part * all >> parts_log, to = (part + 1) * all >> parts_log;
    if (from == to)
        return;
    // the groups in front of the run's first
    const int lane = threadIdx.x & 31, rank = __popc(begins & ((1u << lane) - 1));
    const unsigned left = __ballot_sync(0xffffffffu, (begins >> lane & 1) && (rank + 1) * planes > from);
    const int skipped = (__popc(begins) - __popc(left)) * planes;
    begins = left;
    from -= skipped;
    to -= skipped;
#pragma unroll 1
    for (; to > 0; begins &= begins - 1, from = 0, to -= planes)
        f(__ffs(begins) - 1, from, to < planes ? to : planes);
}

// Keys that are turned.  A team of D threads takes a group, a lane 16 values of one row, so that a lane keeps its pairs'
// sines and cosines, and the turned values, while it goes through the heads with the next one's rows on their way.
template <typename T, int D, bool kHalf>
struct Team {
    static constexpr int kLanes = D / 16, kSize = kGroup * kLanes, kCount = kThreads / kSize, kWarps = kSize / 32;
    const Kv8Append &p;
    const RopeParams &rope;
    uint32_t (*const tops)[kWarps];      // [2] in shared memory: the warps' maxima
    const int team, lane, warp, i, v;    // warp of the team; the lane's row of the group, and its place there
    int turn = 0;                        // tops that the next maximum goes to

    __device__ __forceinline__ void meet() const
    {
        asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(kSize) : "memory");
    }
    // the largest x of all lanes
    __device__ __forceinline__ uint32_t largest(uint32_t x)
    {
        x = __reduce_max_sync(0xffffffffu, x);
        if (lane == 0)
            tops[turn][warp] = x;
        meet();
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            x = max(x, tops[turn][w]);
        turn ^= 1;                       // the next one's writers have met again before they come back to these
        return x;
    }

    // one group's rows of the heads first to end - 1
    __device__ __forceinline__ void group(const Window &w, int l, int first, int end)
    {
        const unsigned rows = w.rows(l);
        const int64_t id = __shfl_sync(0xffffffffu, w.slot, l) >> 4, row = w.first + l + i;
        const int spot = (int)(__shfl_sync(0xffffffffu, w.slot, (l + lane) & 31) & (kGroup - 1));
        const unsigned tokens = __reduce_or_sync(0xffffffffu, (rows >> lane) & 1 ? 1u << spot : 0u);
        const int token = (int)(__shfl_sync(0xffffffffu, w.slot, (l + i) & 31) & (kGroup - 1));
        const bool on = (rows >> i) & 1, anew = tokens & 1, turned = v < rope.pairs / 8;
        int a, b;
        lane_vectors(v, rope.pairs, kHalf, a, b);
        Spins spins;
        const int64_t pos = on ? __ldg(p.pos + row) : 0;
        // the next head's rows, bytes and scale
        const uint4 *from = p.k + row * p.kv_stride + first * (D / 8);
        const int shift = p.cache.page_shift - 4;
        float *scale_next;
        uint8_t *at_next = group_at<D>(p.cache, id >> shift, (int)(id & (((int64_t)1 << shift) - 1)), 2 * first, &scale_next);
        const int64_t at_step = 2 * plane_bytes<D>(p.cache);
        const int scale_step = 2 << shift;
        uint4 next[2];
        float next_old;
        auto fetch = [&]() {
            next[0] = next[1] = make_uint4(0, 0, 0, 0);
            if (on) {
                next[0] = __ldcs(from + a);
                next[1] = __ldcs(from + b);
            }
            next_old = *scale_next;
            from += D / 8;
        };
        fetch();
        if (turned && on) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = spin_of(angle_of(rope.turns[8 * v + 2 * k], pos), rope.gain),
                             g = spin_of(angle_of(rope.turns[8 * v + 2 * k + 1], pos), rope.gain);
                spins.c[k] = ptx::pair(f.x, g.x);
                spins.s[k] = ptx::pair(f.y, g.y);
            }
        }
#pragma unroll 1
        for (int head = first; head < end; ++head) {
            const Pairs in = pairs_of<T, kHalf>(next[0], next[1]);
            const float old = next_old;
            float *const scale_at = scale_next;
            uint8_t *const at = at_next;
            scale_next += scale_step;
            at_next += at_step;
            if (head + 1 < end)
                fetch();
            Pairs x = in;
            if (turned && on)
                hs::kv8::turn(x, spins);
            // element `second` of pair j times f, closely
            auto closely = [&](int j, bool second, float f) {
                auto of = [&](const uint64_t (&z)[4]) {
                    float one[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 w = ptx::unpair(z[k]);
                        one[k] = j & 1 ? w.y : w.x;
                    }
                    const float low = j & 2 ? one[1] : one[0], high = j & 2 ? one[3] : one[2];
                    return j & 4 ? high : low;
                };
                return turned_closely(angle_of(rope.turns[8 * v + j], rope.rest[8 * v + j], pos), Two{rope.gain, rope.gain_low}, of(in.x),
                                      of(in.y), f, second);
            };
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = ptx::unpair(x.x[k]), g = ptx::unpair(x.y[k]);
                top = fmaxf(fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y))), fmaxf(fabsf(g.x), fabsf(g.y)));
            }
            uint32_t bits = largest(__float_as_uint(top));
            const bool odd = bits >= 0x7f800000u;       // an infinity among the values: they become NaN, and do not count
            if (odd) {
                top = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    // turned, both of a pair: beside one that is too large for float32 the other may be rounding alone
                    if (turned)
                        x.x[k] = ptx::fma2(x.y[k], 0, x.x[k]);
                    x.y[k] = ptx::fma2(turned ? x.x[k] : x.y[k], 0, x.y[k]);
                    x.x[k] = ptx::fma2(x.x[k], 0, x.x[k]);
                    const float2 f = ptx::unpair(x.x[k]), g = ptx::unpair(x.y[k]);
                    top = fmaxf(fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y))), fmaxf(fabsf(g.x), fabsf(g.y)));
                }
                bits = largest(__float_as_uint(top));
            }
            int e = exponent_of(bits);
            // |x| + |y| is at most twice the largest turned value, and 2^-20 of that 15 steps
            if (abs((int)(bits & 0x7fffffu) - 0x600000) <= 16) {
                e = (int)(bits >> 23) - 127 - 8;
                const float close = __uint_as_float(bits) * (1.f - 0x1p-18f);
                const float by = inverse(power_of_two(e < -126 ? -126 : e));
                bool above = false;
#pragma unroll 1
                for (int j = 0; j < 16; ++j) {
                    float y = 0.f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float2 f = ptx::unpair(k < 4 ? x.x[k % 4] : x.y[k % 4]);
                        y = k == j >> 1 ? fabsf(j & 1 ? f.y : f.x) : y;
                    }
                    if (!on || !(y >= close))
                        continue;
                    // elements that are not turned are what they are
                    const Two z = turned ? closely(j & 7, j >> 3, by) : Two{y * by, 0.f};
                    above = above || (fabsf(z.high) - 448.f) + (z.high > 0.f ? z.low : -z.low) > 0.f;
                }
                __syncwarp();
                e += largest(above);
            }
            const float need = power_of_two(e < -126 ? -126 : e), scale = anew ? need : fmaxf(old, need),
                        by = inverse(scale);
            if (i == 0 && v == 0)
                *scale_at = scale;
            if (!anew && need > old && !((tokens >> i) & 1)) {
                // what the group holds: token i's bytes
                const float shrink = old / need;
                uint4 *const held = reinterpret_cast<uint4 *>(at + i * D) + v;
                const uint4 y = *held;
                auto again = [&](uint32_t u) {
                    const float2 f = widen<__half>(e4m3_to_f16(u)), h = widen<__half>(e4m3_to_f16_high(u));
                    return to_e4m3(f.x * shrink, f.y * shrink, h.x * shrink, h.y * shrink);
                };
                *held = make_uint4(again(y.x), again(y.y), again(y.z), again(y.w));
            }
            if (on) {
                const uint64_t by2 = ptx::pair(by, by);
                uint32_t byte[4];
                if (turned) {
                    // and two roundings to multiples of 2^-149, where those count
                    const float off = kOff * rope.gain * by, least = by >= 0x1p100f ? by * 0x1p-148f : 0.f;
                    quantise_turned(x, in, by2, ptx::pair(off, off), ptx::pair(least, least), by, top == 0.f, closely, byte);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        x.x[k] = ptx::mul2(x.x[k], by2);
                        x.y[k] = ptx::mul2(x.y[k], by2);
                    }
                    bytes_of<kHalf>(x, byte);
                }
                uint8_t *const to = at + token * D;
                *reinterpret_cast<uint2 *>(to + 8 * a) = make_uint2(byte[0], byte[1]);
                *reinterpret_cast<uint2 *>(to + 8 * b) = make_uint2(byte[2], byte[3]);
            }
            __syncwarp();
        }
    }

    // turned values times by2 as bytes; off2 times |x| + |y| of `in`, and least2, is how far
    // they may be off; zeros: all are
    template <typename Closely>
    __device__ __forceinline__ static void quantise_turned(const Pairs &x, const Pairs &in, uint64_t by2, uint64_t off2,
                                                           uint64_t least2, float by, bool zeros, Closely closely,
                                                           uint32_t (&w)[4])
    {
        constexpr uint64_t kAbs = 0x7fffffff7fffffffull, kSign = 0x8000000080000000ull;
        Pairs low, high;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint64_t off = ptx::fma2(ptx::add2(in.x[k] & kAbs, in.y[k] & kAbs), off2, least2);
            high.x[k] = ptx::fma2(x.x[k], by2, off);
            high.y[k] = ptx::fma2(x.y[k], by2, off);
            low.x[k] = ptx::fma2(x.x[k], by2, off ^ kSign);
            low.y[k] = ptx::fma2(x.y[k], by2, off ^ kSign);
        }
        uint32_t z[4];
        bytes_of<kHalf>(low, w);
        bytes_of<kHalf>(high, z);
        // values that go to two numbers by what they may be off; not -0, to -0 and 0
#pragma unroll 1
        while (!zeros && ((w[0] ^ z[0]) | (w[1] ^ z[1]) | (w[2] ^ z[2]) | (w[3] ^ z[3])) != 0) {
            const uint64_t first = (uint64_t)(w[1] ^ z[1]) << 32 | (w[0] ^ z[0]);
            const int byte = first != 0 ? (__ffsll(first) - 1) / 8
                                        : 8 + (__ffsll((uint64_t)(w[3] ^ z[3]) << 32 | (w[2] ^ z[2])) - 1) / 8;
            const Two q = closely(kHalf ? byte & 7 : byte >> 1, kHalf ? byte >> 3 : byte & 1, by);
            const uint32_t mask = 0xffu << 8 * (byte & 3), put = to_e4m3(toward(q), 0.f, 0.f, 0.f) << 8 * (byte & 3);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k == byte >> 2) {
                    w[k] = (w[k] & ~mask) | put;
                    z[k] = (z[k] & ~mask) | put;
                }
        }
    }
};

// Blocks: the turned keys' teams, which take longest; warps for the other planes' heads; q.  With positions 24 warps share an
// SM (80 registers, a few of them spilled) where four meet for a head, 14,494 rows of 4 x 128 30.6 us, 33.9 with 16 warps;
// 16 where two do, 12,000 rows of 16 x 64 34.8 us, 41.0 with 24.
template <typename T, int D, bool kRope, bool kHalf>
__global__ void __launch_bounds__(kThreads, kRope ? (D == 64 ? 4 : 6) : 8)
kv8_append_kernel(const __grid_constant__ Kv8Append p, const __grid_constant__ RopeParams rope)
{
    using Keys = Team<T, D, kHalf>;
    __shared__ uint32_t tops[Keys::kCount][2][Keys::kWarps];
    pdl_wait_and_release();
    const int lane = threadIdx.x & 31;
    if constexpr (kRope) {
        if ((int)blockIdx.x < p.team_blocks) {
            const int team = threadIdx.x / Keys::kSize, in_team = threadIdx.x % Keys::kSize;
            const int unit = blockIdx.x * Keys::kCount + team, slice = unit / p.windows;
            if (slice >> p.slices_log)
                return;
            const Window w(p, (int64_t)(unit - slice * p.windows) * kGroup, false, lane, [&](int64_t first) {
                // the first two heads that fall to this team where the window begins one group
                const int head = (slice * p.cache.n_kv >> p.slices_log) + in_team / 32;
                if (in_team < 64 && head < (slice + 1) * p.cache.n_kv >> p.slices_log)
                    ahead<D>(p, p.k + head * (D / 8), first, lane);
            });
            Keys keys{p, rope, tops[team], team, lane, in_team / 32, in_team / Keys::kLanes, in_team % Keys::kLanes};
            share(w.begins, p.cache.n_kv, slice, p.slices_log, [&](int l, int from, int to) { keys.group(w, l, from, to); });
            return;
        }
    }
    if ((int)blockIdx.x < p.team_blocks + p.warp_blocks) {
        const int unit = (blockIdx.x - p.team_blocks) * (kThreads / 32) + threadIdx.x / 32, part = unit / p.windows;
        const int planes = (kRope ? 1 : 2) * p.cache.n_kv;            // values alone, or both planes of each head
        if (part >> p.parts_log)
            return;
        const Window w(p, (int64_t)(unit - part * p.windows) * kGroup, part == 0, lane, [&](int64_t first) {
            // the plane that falls to this warp where the window begins one group
            const int plane = part * planes >> p.parts_log;
            if (plane < (part + 1) * planes >> p.parts_log)
                ahead<D>(p, (kRope || (plane & 1) ? p.v : p.k) + (kRope ? plane : plane >> 1) * (D / 8), first, lane);
        });
        const int shift = p.cache.page_shift - 4;
        share(w.begins, planes, part, p.parts_log, [&](int l, int from, int to) {
            const int64_t id = __shfl_sync(0xffffffffu, w.slot, l) >> 4;
            Group g;
            g.rows = w.rows(l);
            g.spot = (int)(__shfl_sync(0xffffffffu, w.slot, (l + lane) & 31) & (kGroup - 1));
            g.tokens = __reduce_or_sync(0xffffffffu, (g.rows >> lane) & 1 ? 1u << g.spot : 0u);
#pragma unroll 1
            for (int x = from; x < to; ++x) {
                const int head_plane = kRope ? 2 * x + 1 : x;
                g.at = group_at<D>(p.cache, id >> shift, (int)(id & (((int64_t)1 << shift) - 1)), head_plane, &g.scale_at);
                g.old = *g.scale_at;
                quantise<T, D>(g, (head_plane & 1 ? p.v : p.k) + (w.first + l) * p.kv_stride + (head_plane >> 1) * (D / 8),
                               p.kv_stride, lane);
            }
        });
        return;
    }
    if constexpr (kRope) {
        const RopeRows q{p.q, nullptr, p.q_out, nullptr, p.q_stride, 0, p.q_out_stride, 0, p.pos, p.n_rows, p.n_heads, 0, p.q_slices};
        turn_rows<T, D, kHalf>(q, rope, p.slots,
                               (int64_t)(blockIdx.x - p.team_blocks - p.warp_blocks) * (kThreads / Keys::kLanes));
    }
}

// the logarithm of how many share up to `all` jobs of each of `windows` windows so that there are `wanted` in all
int32_t shared_by(int32_t all, int32_t windows, int64_t wanted)
{
    int32_t log = 0;
    while (1 << log < all && (int64_t)windows << log < wanted)
        ++log;
    return log;
}

template <typename T, int D>
cudaError_t launch(Kv8Append p, const RopeParams *rope, int sm_count, cudaStream_t s)
{
    constexpr int kTeams = kThreads / D, kJobs = kThreads / (D / 16);
    constexpr int64_t most = INT32_MAX / 4;
    p.windows = (int)((p.n_rows + kGroup - 1) / kGroup);
    // 24 warps for each SM (256 rows of 8 x 128, each a group, 4.3 us), or more: one for each plane of a prompt's group
    // (28,913 rows 29.5 us; 34.2 with fewer, which wait for one group's rows after another).  Beside turned keys, whose teams
    // are the longer part and share the SM, four (256 rows 7.0 us, 7.4 with eight), or one for each two heads
    // (12,000 rows of 16 + 16 x 128 51.6 us, 63.8 with eight).
    const int planes = (rope != nullptr ? 1 : 2) * p.cache.n_kv;
    int64_t warps = (int64_t)sm_count * (rope != nullptr ? 4 : 24);
    const int64_t prompt = (int64_t)p.windows * (rope != nullptr ? (planes + 1) / 2 : planes);
    warps = prompt > warps ? prompt : warps;
    p.parts_log = shared_by(kGroup * planes, p.windows, warps < most ? warps : most);
    p.warp_blocks = ((p.windows << p.parts_log) + kThreads / 32 - 1) / (kThreads / 32);
    int64_t blocks = p.warp_blocks;
    if (rope != nullptr) {
        // Teams of up to 8 heads, so that sines and cosines are worth it (14,494 rows of 4 heads 30.6 us, 32.4 with 2 to
        // a team) and the last wave stays short (12,000 rows of 16 heads 51.6 us, 59.2 with all in a team); of
        // fewer where there are not two to an SM (2,000 rows of 8 heads 10.7 us so, 12.0 with four, 12.1 with one).
        const int64_t eights = (int64_t)p.windows * ((p.cache.n_kv + 7) / 8);
        int64_t teams = (int64_t)sm_count * 2 * kTeams;
        teams = eights > teams ? eights : teams;
        p.slices_log = shared_by(kGroup * p.cache.n_kv, p.windows, teams < most ? teams : most);
        p.team_blocks = ((p.windows << p.slices_log) + kTeams - 1) / kTeams;
        blocks += p.team_blocks;
        if (p.q != nullptr) {
            p.q_slices = rope_slices(p.n_rows, p.n_heads, sm_count, kJobs);
            blocks += (p.n_rows * p.q_slices + kJobs - 1) / kJobs;
        }
    }
    if (blocks > INT32_MAX)
        return cudaErrorInvalidValue;
    if (rope == nullptr)
        return launch_pdl(kv8_append_kernel<T, D, false, false>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p,
                          RopeParams{});
    return launch_pdl(rope->layout == HS_ROPE_HALF ? kv8_append_kernel<T, D, true, true>
                                                   : kv8_append_kernel<T, D, true, false>,
                      dim3((unsigned)blocks), dim3(kThreads), 0, s, p, *rope);
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
