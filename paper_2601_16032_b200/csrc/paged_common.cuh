// Shared by the kernels around the paged cache: division by a run-time constant, the cache as kernels see it, 16-bit pairs.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "ptx.cuh"

namespace sawtooth {

// n / d for 0 <= n < 2^31 by one multiplication: with l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1 the quotient
// is (mulhi(n, m) + n) >> l (Granlund and Montgomery, "Division by Invariant Integers using Multiplication", 1994).
struct FastDiv {
    uint32_t d = 1, m = 1, l = 0;
    FastDiv() = default;
    explicit FastDiv(uint32_t divisor) : d(divisor) {
        l = 0;
        while ((1ull << l) < divisor) ++l;
        m = (uint32_t)(((1ull << 32) * ((1ull << l) - divisor)) / divisor + 1);
    }
    __host__ __device__ uint32_t div(uint32_t n) const {
#ifdef __CUDA_ARCH__
        return (__umulhi(n, m) + n) >> l;
#else
        return ((uint32_t)(((uint64_t)n * m) >> 32) + n) >> l;
#endif
    }
};

struct CacheView {
    const uint16_t* k;
    const uint16_t* v;
    long long page_stride, token_stride, head_stride;
    long long num_pages;
    FastDiv page;   // page.d = tokens per page
};

__device__ __forceinline__ void note_index(int* status, int code) { atomicCAS(status, 0, code); }

// The kernels here are launched before the previous one of the stream has ended.  Until all that it wrote can be seen no thread reads or
// writes global memory, and since every thread waits, a kernel that has ended leaves none behind it that still runs.
__device__ __forceinline__ void previous_kernel_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes)   // copies `bytes` (16 or 0), zero-fills the rest
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

// Clusters: reading the shared memory of the other CTAs.
__device__ __forceinline__ uint32_t in_cta(uint32_t smem_addr, int rank)       // the same place in another CTA of the cluster
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr), "r"(rank));
    return a;
}
__device__ __forceinline__ float ld_cluster1(uint32_t a)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t a)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <int kBf16>
__device__ __forceinline__ void unpack2(uint32_t u, float& lo, float& hi) {
    if (kBf16) {
        lo = __uint_as_float(u << 16);
        hi = __uint_as_float(u & 0xffff0000u);
    } else {
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(u));
    }
}

}  // namespace sawtooth
