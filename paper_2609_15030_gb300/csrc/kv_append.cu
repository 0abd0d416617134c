// New tokens' K and V rows of one layer into their pages (the attention entries of the recomputed
// suffix, Section 2.2 of the paper, and of each decode step).
//
// A copy: row r's n_kv * d keys go to row slot % P of plane 0 of block slot / P and its values to
// the same row of plane 1, both contiguous runs.
#include "attn_internal.cuh"

namespace hs {
namespace {

constexpr int kThreads = 256;

__global__ void __launch_bounds__(kThreads)
kv_append_kernel(const uint4 *k, const uint4 *v, int64_t stride_vecs, const int64_t *slots,
                 int64_t n_rows, uint4 *cache, int32_t row_vecs, int32_t page_shift,
                 int64_t num_blocks, int32_t *d_err)
{
    pdl_wait_and_release();
    const int64_t page_mask = ((int64_t)1 << page_shift) - 1;
    const int64_t units = n_rows * 2 * row_vecs;
    for (int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x; u < units;
         u += (int64_t)gridDim.x * kThreads) {
        const int64_t plane_row = u / row_vecs;
        const int32_t x = (int32_t)(u - plane_row * row_vecs);
        const int64_t r = plane_row >> 1;
        const int plane = (int)(plane_row & 1);
        const int64_t slot = slots[r];
        if (slot < 0)
            continue;
        const int64_t blk = slot >> page_shift;
        if (blk >= num_blocks) {
            if (x == 0 && plane == 0)
                report(d_err, HS_DEVERR_BLOCK_OOB);
            continue;
        }
        const int64_t row = ((blk * 2 + plane) << page_shift) + (slot & page_mask);
        cache[row * row_vecs + x] = (plane ? v : k)[r * stride_vecs + x];
    }
}

}  // namespace

cudaError_t launch_kv_append(const void *k, const void *v, int64_t kv_stride, const int64_t *slots,
                             int64_t n_rows, void *cache, int32_t row_vecs, int32_t page_shift,
                             int64_t num_blocks, int32_t *d_err, int sm_count, cudaStream_t s)
{
    const int64_t units = n_rows * 2 * row_vecs;
    int64_t grid = (units + kThreads - 1) / kThreads;
    const int64_t most = (int64_t)sm_count * 8 * 4;
    if (grid > most)
        grid = most;
    return launch_pdl(kv_append_kernel, dim3((unsigned)grid), dim3(kThreads), 0, s,
                      static_cast<const uint4 *>(k), static_cast<const uint4 *>(v), kv_stride / 8,
                      slots, n_rows, static_cast<uint4 *>(cache), row_vecs, page_shift, num_blocks,
                      d_err);
}

}  // namespace hs
