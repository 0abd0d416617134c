// C-ABI entry points of the rotary positions and the 8-bit cache: host-side validation, then the launches.
// Validation happens before any CUDA runtime call, so argument errors are reported without
// touching the GPU.
#include <cmath>
#include <cstring>

#include "hs_test.h"
#include "kv8_internal.cuh"

namespace {

constexpr double kTurn = 6.283185307179586476925286766559;

inline bool misaligned(const void *p, unsigned by)
{
    return (reinterpret_cast<uintptr_t>(p) & (by - 1)) != 0;
}

inline hs_status cuda_status(cudaError_t e)
{
    return e == cudaSuccess ? HS_OK : HS_ERR_CUDA;
}

inline bool positive(double x)
{
    return x > 0.0 && std::isfinite(x);
}

// its products with 2^-21 and a scale's inverse, 2^126 at most, have to be finite in 32 bits
inline bool usable_amplitude(double x)
{
    return x >= 0x1p-20 && x <= 0x1p20;
}

// 1 / (2 pi), in units of 2^-192, the lowest word first
constexpr uint64_t kTurnsPerRadian[3] = {0x36d8a5664f10e410ull, 0x7f09d5f47d4d3770ull, 0x28be60db9391054aull};

// theta / (2 pi) modulo 1, in units of 2^-96 and to half of one, for |theta| < 2^64: theta is m 2^(e - 53) with integers m and
// e, so that its product with the constant is one of integers.
void turns_of(double theta, uint64_t &turns, int32_t &rest)
{
    using uint128 = unsigned __int128;
    int e;
    const uint64_t m = (uint64_t)std::ldexp(std::frexp(std::fabs(theta), &e), 53);
    uint64_t product[6] = {};
    uint128 carry = 0;
    for (int i = 0; i < 3; ++i) {
        carry += (uint128)m * kTurnsPerRadian[i];
        product[i] = (uint64_t)carry;
        carry >>= 64;
    }
    product[3] = (uint64_t)carry;
    // from units of 2^(e - 53 - 192) to 2^-96
    const int down = 149 - e;
    uint128 x = 0;
    if (down < 256) {
        auto bits = [&](int at) {                    // 64 of the product's
            const int word = at / 64, shift = at % 64;
            return shift == 0 ? product[word] : product[word] >> shift | product[word + 1] << (64 - shift);
        };
        x = (uint128)(down < 192 ? bits(down + 64) : 0) << 64 | bits(down);
        x += bits(down - 1) & 1;
    }
    if (theta < 0.0)
        x = -x;
    x += (uint128)1 << 31;
    turns = (uint64_t)(x >> 32);
    rest = (int32_t)((uint32_t)x - (1u << 31));
}

hs_status check_rope(const hs_rope *rope, int32_t head_dim, hs::RopeParams &p)
{
    if (rope == nullptr || (rope->layout != HS_ROPE_HALF && rope->layout != HS_ROPE_INTERLEAVED) ||
        rope->dims < 1 || rope->dims > head_dim || !usable_amplitude(rope->amplitude))
        return HS_ERR_INVALID_ARG;
    if (rope->dims % 16 != 0)
        return HS_ERR_UNSUPPORTED;
    std::memset(&p, 0, sizeof p);
    p.gain = (float)rope->amplitude;
    p.gain_low = (float)(rope->amplitude - p.gain);
    p.pairs = rope->dims / 2;
    p.layout = rope->layout;
    for (int i = 0; i < p.pairs; ++i) {
        if (!(std::fabs(rope->theta[i]) < 0x1p64))
            return HS_ERR_INVALID_ARG;
        turns_of(rope->theta[i], p.turns[i], p.rest[i]);
    }
    return HS_OK;
}

// a row stride in elements, 0 meaning rows that touch
hs_status check_stride(int64_t stride, int64_t inner)
{
    if (stride < 0 || (stride != 0 && stride < inner))
        return HS_ERR_INVALID_ARG;
    return stride % 8 != 0 ? HS_ERR_MISALIGNED : HS_OK;
}

inline int64_t vectors(int64_t stride, int64_t inner)
{
    return (stride != 0 ? stride : inner) / 8;
}

// what the calls with query heads ask of them
hs_status check_heads(const hs_attn_shape &s)
{
    if (s.n_heads < 1 || s.n_heads % s.n_kv_heads != 0)
        return HS_ERR_INVALID_ARG;
    return s.n_heads / s.n_kv_heads > 128 ? HS_ERR_UNSUPPORTED : HS_OK;
}

int64_t block_bytes(const hs_attn_shape &s)
{
    const int64_t planes = 2 * (int64_t)s.n_kv_heads;
    return (planes * ((int64_t)s.page_size * s.head_dim + s.page_size / HS_KV8_GROUP * 4) + 127) / 128 * 128;
}

hs::Kv8Cache cache_of(const hs_attn_shape &s, const void *cache)
{
    return {static_cast<uint8_t *>(const_cast<void *>(cache)), block_bytes(s), s.num_blocks, s.n_kv_heads,
            hs::attn_page_shift(s.page_size)};
}

hs_status append(const hs_attn_shape *shp, const hs_rope *rope, bool with_rope, const void *q, const void *k,
                 const void *v, int64_t in_stride, const int64_t *pos, const int64_t *slots, int64_t n_rows,
                 void *q_out, int64_t q_out_stride, void *cache, int32_t *d_err, cudaStream_t stream)
{
    if (shp == nullptr || n_rows < 0)
        return HS_ERR_INVALID_ARG;
    const hs_attn_shape s = *shp;
    hs_status st = hs::check_attn_cache(s);
    if (st != HS_OK)
        return st;
    const int64_t inner = (int64_t)s.n_kv_heads * s.head_dim, q_inner = (int64_t)s.n_heads * s.head_dim;
    const bool with_q = with_rope && (q != nullptr || q_out != nullptr);
    if (with_q)
        st = check_heads(s);
    if (st == HS_OK)
        st = check_stride(in_stride, with_q && q_inner > inner ? q_inner : inner);
    if (st == HS_OK && with_q)
        st = check_stride(q_out_stride, q_inner);
    hs::RopeParams params;
    if (st == HS_OK && with_rope)
        st = check_rope(rope, s.head_dim, params);
    if (st != HS_OK || n_rows == 0)
        return st;
    if (n_rows > INT32_MAX)
        return HS_ERR_UNSUPPORTED;
    if (k == nullptr || v == nullptr || slots == nullptr || cache == nullptr || (with_rope && pos == nullptr) ||
        (with_q && (q == nullptr || q_out == nullptr)))
        return HS_ERR_INVALID_ARG;
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(cache, 16) || misaligned(slots, 8) ||
        (with_rope && misaligned(pos, 8)) || (with_q && (misaligned(q, 16) || misaligned(q_out, 16))))
        return HS_ERR_MISALIGNED;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st != HS_OK)
        return st;
    hs::Kv8Append a;
    std::memset(&a, 0, sizeof a);
    a.cache = cache_of(s, cache);
    a.k = static_cast<const uint4 *>(k);
    a.v = static_cast<const uint4 *>(v);
    a.kv_stride = vectors(in_stride, inner);
    a.slots = slots;
    a.n_rows = n_rows;
    a.d_err = d_err;
    if (with_rope)
        a.pos = pos;
    if (with_q) {
        a.q = static_cast<const uint4 *>(q);
        a.q_out = static_cast<uint4 *>(q_out);
        a.q_stride = vectors(in_stride, q_inner);
        a.q_out_stride = vectors(q_out_stride, q_inner);
        a.n_heads = s.n_heads;
    }
    return cuda_status(hs::launch_kv8_append(a, with_rope ? &params : nullptr, s.head_dim, s.dtype, sms, stream));
}

hs_status check_decode(const hs_attn_shape *shp, int64_t max_kv_len, hs::AttnParams &p)
{
    const hs_status st = hs::check_attn_decode(shp, 0, max_kv_len, p);
    // the cache's rows of 128 bytes are counted in 31 bits
    return st == HS_OK && shp->num_blocks > INT32_MAX / (block_bytes(*shp) / 128) ? HS_ERR_UNSUPPORTED : st;
}

hs_status decode(const hs_attn_shape *shp, const void *q, const void *cache, const int32_t *block_table,
                 const int32_t *kv_len, int64_t max_kv_len, void *o, float *lse, void *workspace,
                 int64_t workspace_bytes, int32_t *d_err, cudaStream_t stream, bool stall_for_test)
{
    hs::AttnParams p;
    hs_status st = check_decode(shp, max_kv_len, p);
    if (st != HS_OK || p.batch == 0)
        return st;
    if (kv_len == nullptr)
        return HS_ERR_INVALID_ARG;
    if (misaligned(kv_len, 4))
        return HS_ERR_MISALIGNED;
    p.q = q;
    p.cache = cache;
    p.table = block_table;
    p.kv_len = kv_len;
    p.o = o;
    p.lse = lse;
    p.d_err = d_err;
    p.stall_for_test = stall_for_test;
    st = hs::check_attn_pointers(p, workspace, workspace_bytes);
    if (st != HS_OK)
        return st;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    hs::Kv8Plan plan;
    if (st == HS_OK)
        st = hs::attn_workspace(hs::plan_kv8_decode(p, plan, shp->head_dim, sms), workspace, workspace_bytes, p);
    if (st != HS_OK)
        return st;
    return cuda_status(hs::launch_kv8_decode(p, plan, cache_of(*shp, cache), shp->head_dim, shp->dtype, stream));
}

}  // namespace

extern "C" {

hs_status hs_rope_plan(int32_t dims, int32_t layout, double base, int32_t scaling, double factor,
                       int64_t context, double low, double high, double amplitude, hs_rope *out)
{
    const bool by_turns = scaling == HS_ROPE_TURNS || scaling == HS_ROPE_INDEX;
    if (out == nullptr || dims < 1 || (layout != HS_ROPE_HALF && layout != HS_ROPE_INTERLEAVED) ||
        scaling < HS_ROPE_PLAIN || scaling > HS_ROPE_INDEX || !positive(base) || base <= 1.0 ||
        !usable_amplitude(amplitude) || (scaling != HS_ROPE_PLAIN && !(positive(factor) && factor >= 1.0)) ||
        (by_turns && (context < 1 || !positive(low) || !positive(high) || low >= high)))
        return HS_ERR_INVALID_ARG;
    if (dims % 16 != 0 || dims > 2 * HS_ROPE_MAX_PAIRS)
        return HS_ERR_UNSUPPORTED;
    if (scaling == HS_ROPE_BASE) {
        base *= std::pow(factor, (double)dims / (dims - 2));
        if (!std::isfinite(base))
            return HS_ERR_INVALID_ARG;
    }
    hs_rope r;
    std::memset(&r, 0, sizeof r);
    r.dims = dims;
    r.layout = layout;
    r.amplitude = amplitude;
    double first = 0.0, last = 0.0;              // HS_ROPE_INDEX: where the share begins to fall, and ends
    if (scaling == HS_ROPE_INDEX) {
        auto index = [&](double turns) {
            return dims * std::log((double)context / (turns * kTurn)) / (2.0 * std::log(base));
        };
        first = std::fmax(std::floor(index(high)), 0.0);
        last = std::fmin(std::ceil(index(low)), dims - 1.0);
    }
    for (int i = 0; i < dims / 2; ++i) {
        const double theta = std::pow(base, -2.0 * i / dims);
        double share = 1.0;                      // of the angle that is not divided
        if (scaling == HS_ROPE_LINEAR)
            share = 0.0;
        else if (scaling == HS_ROPE_TURNS)
            share = ((double)context * theta / kTurn - low) / (high - low);
        else if (scaling == HS_ROPE_INDEX)
            share = 1.0 - (i - first) / std::fmax(last - first, 0.001);
        share = share < 0.0 ? 0.0 : share > 1.0 ? 1.0 : share;
        r.theta[i] = share == 1.0 ? theta : theta * share + theta / factor * (1.0 - share);
    }
    *out = r;
    return HS_OK;
}

hs_status hs_rope_apply(const hs_attn_shape *shp, const hs_rope *rope, const void *q, const void *k,
                        int64_t in_stride, const int64_t *pos, int64_t n_rows, void *q_out,
                        int64_t q_out_stride, void *k_out, int64_t k_out_stride, cudaStream_t stream)
{
    if (shp == nullptr || n_rows < 0)
        return HS_ERR_INVALID_ARG;
    const hs_attn_shape s = *shp;
    if (s.n_kv_heads < 1 || (s.dtype != HS_BF16 && s.dtype != HS_FP16))
        return HS_ERR_INVALID_ARG;
    hs_status st = check_heads(s);
    if (st == HS_ERR_INVALID_ARG)
        return st;
    if (st != HS_OK || (s.head_dim != 64 && s.head_dim != 128) || s.n_kv_heads > 1024)
        return HS_ERR_UNSUPPORTED;
    hs::RopeParams params;
    st = check_rope(rope, s.head_dim, params);
    if (st != HS_OK)
        return st;
    const int64_t q_inner = (int64_t)s.n_heads * s.head_dim, k_inner = (int64_t)s.n_kv_heads * s.head_dim;
    if ((q == nullptr && k == nullptr && n_rows > 0) || (q == nullptr) != (q_out == nullptr) ||
        (k == nullptr) != (k_out == nullptr))
        return HS_ERR_INVALID_ARG;
    st = check_stride(in_stride, q != nullptr ? q_inner : k_inner);
    if (st == HS_OK && q != nullptr)
        st = check_stride(q_out_stride, q_inner);
    if (st == HS_OK && k != nullptr)
        st = check_stride(k_out_stride, k_inner);
    if (st != HS_OK || n_rows == 0)
        return st;
    if (n_rows > INT32_MAX)
        return HS_ERR_UNSUPPORTED;
    if (pos == nullptr)
        return HS_ERR_INVALID_ARG;
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(q_out, 16) || misaligned(k_out, 16) ||
        misaligned(pos, 8))
        return HS_ERR_MISALIGNED;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st != HS_OK)
        return st;
    hs::RopeRows r;
    std::memset(&r, 0, sizeof r);
    r.q = static_cast<const uint4 *>(q);
    r.k = static_cast<const uint4 *>(k);
    r.q_out = static_cast<uint4 *>(q_out);
    r.k_out = static_cast<uint4 *>(k_out);
    r.q_stride = vectors(in_stride, q_inner);
    r.k_stride = vectors(in_stride, k_inner);
    r.q_out_stride = vectors(q_out_stride, q_inner);
    r.k_out_stride = vectors(k_out_stride, k_inner);
    r.pos = pos;
    r.n_rows = n_rows;
    r.n_heads = q != nullptr ? s.n_heads : 0;
    r.n_kv = k != nullptr ? s.n_kv_heads : 0;
    return cuda_status(hs::launch_rope(r, params, s.head_dim, s.dtype, sms, stream));
}

hs_status hs_kv8_block_bytes(const hs_attn_shape *shp, int64_t *bytes_out)
{
    if (shp == nullptr || bytes_out == nullptr)
        return HS_ERR_INVALID_ARG;
    const hs_status st = hs::check_attn_cache(*shp);
    if (st == HS_OK)
        *bytes_out = block_bytes(*shp);
    return st;
}

hs_status hs_kv8_append(const hs_attn_shape *shp, const void *k, const void *v, int64_t kv_stride,
                        const int64_t *slots, int64_t n_rows, void *cache, int32_t *d_err,
                        cudaStream_t stream)
{
    return append(shp, nullptr, false, nullptr, k, v, kv_stride, nullptr, slots, n_rows, nullptr, 0, cache, d_err,
                  stream);
}

hs_status hs_kv8_append_rope(const hs_attn_shape *shp, const hs_rope *rope, const void *q, const void *k,
                             const void *v, int64_t in_stride, const int64_t *pos, const int64_t *slots,
                             int64_t n_rows, void *q_out, int64_t q_out_stride, void *cache,
                             int32_t *d_err, cudaStream_t stream)
{
    return append(shp, rope, true, q, k, v, in_stride, pos, slots, n_rows, q_out, q_out_stride, cache, d_err,
                  stream);
}

hs_status hs_kv8_decode(const hs_attn_shape *shp, const void *q, const void *cache,
                        const int32_t *block_table, const int32_t *kv_len, int64_t max_kv_len, void *o,
                        float *lse, void *workspace, int64_t workspace_bytes, int32_t *d_err,
                        cudaStream_t stream)
{
    return decode(shp, q, cache, block_table, kv_len, max_kv_len, o, lse, workspace, workspace_bytes, d_err, stream,
                  false);
}

hs_status hs_test_kv8_stalled(const hs_attn_shape *shp, const void *q, const void *cache,
                              const int32_t *block_table, const int32_t *kv_len, int64_t max_kv_len,
                              void *o, float *lse, void *workspace, int64_t workspace_bytes,
                              int32_t *d_err, cudaStream_t stream)
{
    return decode(shp, q, cache, block_table, kv_len, max_kv_len, o, lse, workspace, workspace_bytes, d_err, stream,
                  true);
}

hs_status hs_kv8_decode_workspace_bytes(const hs_attn_shape *shp, int64_t max_kv_len, int64_t *bytes_out)
{
    if (bytes_out == nullptr)
        return HS_ERR_INVALID_ARG;
    hs::AttnParams p;
    hs_status st = check_decode(shp, max_kv_len, p);
    if (st != HS_OK)
        return st;
    *bytes_out = 0;
    if (p.batch == 0)
        return HS_OK;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st != HS_OK)
        return st;
    hs::Kv8Plan plan;
    const int64_t need = hs::plan_kv8_decode(p, plan, shp->head_dim, sms);
    if (need < 0)
        return HS_ERR_UNSUPPORTED;
    *bytes_out = need;
    return HS_OK;
}

hs_status hs_kv8_read(const hs_attn_shape *shp, const void *cache, const int32_t *block_table,
                      const int32_t *kv_len, int64_t max_kv_len, void *out, int64_t out_blocks,
                      const int32_t *out_table, int32_t *d_err, cudaStream_t stream)
{
    if (shp == nullptr)
        return HS_ERR_INVALID_ARG;
    const hs_attn_shape s = *shp;
    hs_status st = hs::check_attn_cache(s);
    if (st == HS_ERR_INVALID_ARG)
        return st;
    const int64_t room = s.max_pages > INT32_MAX ? INT64_MAX : s.max_pages * s.page_size;
    if (s.batch < 0 || s.max_pages < 0 || max_kv_len < 0 || max_kv_len > room || out_blocks < 0)
        return HS_ERR_INVALID_ARG;
    if (st != HS_OK)
        return st;
    if (s.batch > HS_MAX_BATCH || max_kv_len > INT32_MAX - 8192 ||
        s.batch * ((max_kv_len + HS_KV8_GROUP - 1) / HS_KV8_GROUP) > INT32_MAX)
        return HS_ERR_UNSUPPORTED;
    if (s.batch == 0 || max_kv_len == 0)
        return HS_OK;
    if (cache == nullptr || block_table == nullptr || kv_len == nullptr || out == nullptr || out_table == nullptr ||
        s.num_blocks < 1 || out_blocks < 1)
        return HS_ERR_INVALID_ARG;
    if (misaligned(cache, 16) || misaligned(out, 16) || misaligned(block_table, 4) || misaligned(out_table, 4) ||
        misaligned(kv_len, 4))
        return HS_ERR_MISALIGNED;
    int sms = 0;
    st = hs::device_sm_count(&sms);
    if (st != HS_OK)
        return st;
    hs::Kv8Read r;
    std::memset(&r, 0, sizeof r);
    r.cache = cache_of(s, cache);
    r.table = block_table;
    r.out_table = out_table;
    r.kv_len = kv_len;
    r.out = static_cast<uint4 *>(out);
    r.out_blocks = out_blocks;
    r.max_pages = s.max_pages;
    r.d_err = d_err;
    r.batch = s.batch;
    r.max_kv = (int32_t)max_kv_len;
    return cuda_status(hs::launch_kv8_read(r, s.head_dim, s.dtype, sms, stream));
}

}  // extern "C"
