// cluster.cuh -- blocks of a cluster: barrier, reads and writes of each other's
// shared memory, and an mbarrier that blocks arrive at in each other.
#pragma once

#include "tc.cuh"

namespace lrc {
namespace cl {

__device__ __forceinline__ uint32_t size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Every thread of every block of the cluster.
__device__ __forceinline__ void sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The place of p in the shared memory of block `rank`.
__device__ __forceinline__ uint32_t place(const void* p, uint32_t rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ float4 load4(const float* p, uint32_t rank) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(place(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void store(float* p, uint32_t rank, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(place(p, rank)), "f"(v) : "memory");
}
// Arrives at block rank's barrier: what the thread has written before is there for
// those who wait with wait().
__device__ __forceinline__ void arrive(uint64_t* bar, uint32_t rank) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(place(bar, rank)) : "memory");
}
// Waits for the phase; after tc::kWaitLimitNs records `code` in *err and raises *abort.
__device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity, volatile int* abort, unsigned int* err,
                                     unsigned int code) {
    const uint64_t t0 = tc::globaltimer();
    while (true) {
        uint32_t ok;
        asm volatile(
            "{\n .reg .pred p;\n"
            " mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
            " selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok) : "r"(tc::smem_u32(bar)), "r"(parity) : "memory");
        if (ok || *abort) return;
        if (tc::globaltimer() - t0 > tc::kWaitLimitNs) {
            atomicOr(err, code);
            *abort = 1;
            return;
        }
    }
}

}  // namespace cl
}  // namespace lrc
