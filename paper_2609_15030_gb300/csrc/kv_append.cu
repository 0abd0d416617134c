// New tokens' K and V rows of one layer into their pages (the attention entries of the recomputed
// suffix, Section 2.2 of the paper, and of each decode step).
//
// A copy: row r's n_kv * d keys go to row slot % P of plane 0 of block slot / P and its values to
// the same row of plane 1, both contiguous runs.
#include "attn_internal.cuh"

namespace hs {
namespace {

constexpr int kThreads = 256;
// rows that a block takes at a time, so that a vector's place among them is a small number
template <int kUnroll>
__host__ __device__ __forceinline__ int32_t rows_at_once(int32_t row_vecs)
{
    const int32_t n = kThreads * kUnroll / (2 * row_vecs);
    return n > 0 ? n : 1;
}

// kUnroll 16-byte vectors per thread in flight before the first store.  The rows of k and v are streamed
// (nothing reads them again), the pages written through the cache, where the attention finds them.
// Bound by HBM where there are many rows: 38,656 rows of 8 x 128 keys and values (317 MB) take 48.6 us,
// 6.5 TB/s, with four vectors and 53 us with one; a decode step's 32 rows of 4 x 128 take 1.6 us with
// one and 2.1 with four, which spread over a quarter of the blocks.
template <int kUnroll>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const uint4 *k, const uint4 *v, int64_t stride_vecs, const int64_t *slots,
                 int64_t n_rows, uint4 *cache, const __grid_constant__ Divisor row_vecs,
                 int32_t page_shift, int64_t num_blocks, int32_t *d_err)
{
    pdl_wait_and_release();
    const int64_t page_mask = ((int64_t)1 << page_shift) - 1;
    const int32_t rows = rows_at_once<kUnroll>(row_vecs.d), vecs = rows * 2 * row_vecs.d;
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < n_rows; r0 += (int64_t)gridDim.x * rows) {
        for (int32_t i0 = threadIdx.x; i0 < vecs; i0 += kThreads * kUnroll) {
            uint4 y[kUnroll];
            uint4 *to[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int32_t i = i0 + u * kThreads;
                const int32_t plane_row = row_vecs.div(i), x = i - plane_row * row_vecs.d;
                const int64_t r = r0 + (plane_row >> 1);
                const int plane = plane_row & 1;
                to[u] = nullptr;
                y[u] = make_uint4(0, 0, 0, 0);
                if (i >= vecs || r >= n_rows)
                    continue;
                const int64_t slot = __ldg(slots + r);
                y[u] = __ldcs((plane ? v : k) + r * stride_vecs + x);
                if (slot < 0)
                    continue;
                const int64_t blk = slot >> page_shift;
                if (blk >= num_blocks) {
                    if (x == 0 && plane == 0)
                        report(d_err, HS_DEVERR_BLOCK_OOB);
                    continue;
                }
                to[u] = cache + (((blk * 2 + plane) << page_shift) + (slot & page_mask)) * row_vecs.d + x;
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                if (to[u] != nullptr)
                    *to[u] = y[u];
        }
    }
}

template <int kUnroll>
cudaError_t launch(const void *k, const void *v, int64_t kv_stride, const int64_t *slots, int64_t n_rows,
                   void *cache, int32_t row_vecs, int32_t page_shift, int64_t num_blocks, int32_t *d_err,
                   int sm_count, cudaStream_t s)
{
    Divisor by;
    by.set(row_vecs);
    const int64_t each = rows_at_once<kUnroll>(row_vecs);
    int64_t grid = (n_rows + each - 1) / each;
    const int64_t most = (int64_t)sm_count * 8 * 4;
    if (grid > most)
        grid = most;
    return launch_pdl(kv_append_kernel<kUnroll>, dim3((unsigned)grid), dim3(kThreads), 0, s,
                      static_cast<const uint4 *>(k), static_cast<const uint4 *>(v), kv_stride / 8,
                      slots, n_rows, static_cast<uint4 *>(cache), by, page_shift, num_blocks, d_err);
}

}  // namespace

cudaError_t launch_kv_append(const void *k, const void *v, int64_t kv_stride, const int64_t *slots,
                             int64_t n_rows, void *cache, int32_t row_vecs, int32_t page_shift,
                             int64_t num_blocks, int32_t *d_err, int sm_count, cudaStream_t s)
{
    // one vector per thread while that does not fill the SMs' eight blocks
    const bool few = n_rows * 2 * row_vecs <= (int64_t)sm_count * 8 * kThreads;
    return (few ? launch<1> : launch<4>)(k, v, kv_stride, slots, n_rows, cache, row_vecs, page_shift,
                                         num_blocks, d_err, sm_count, s);
}

}  // namespace hs
