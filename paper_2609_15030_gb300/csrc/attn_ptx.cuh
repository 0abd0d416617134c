// Inline-PTX wrappers that the attention kernel uses beside those of sm100_ptx.cuh: register shares of
// warpgroups, four-dimensional TMA loads, asynchronous copies, paired additions, bf16 products.
#pragma once

#include "sm100_ptx.cuh"

namespace hs {
namespace ptx {

// registers per thread of this warpgroup (all four of its warps), out of those the block was launched with
template <int N>
__device__ __forceinline__ void more_registers()
{
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

template <int N>
__device__ __forceinline__ void fewer_registers()
{
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *tmap, int32_t x, int32_t y,
                                            int32_t z, int32_t w, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void prefetch_tensormap(const void *tmap)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tmap)) : "memory");
}

// 16 bytes of global memory to shared memory
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

__device__ __forceinline__ void cp_async_wait_all()
{
    asm volatile("cp.async.wait_all;" ::: "memory");
}

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// idesc_f16 with bf16 A and B (format 1)
__host__ __device__ constexpr uint32_t idesc_bf16(int M, int N, int b_mn = 0)
{
    return idesc_f16(M, N, b_mn) | (1u << 7) | (1u << 10);
}

}  // namespace ptx
}  // namespace hs
