// Clusters: rank, barrier, stores to a peer's shared memory. Only for
// launches with a cluster dimension: without one these stores are illegal instructions.
#pragma once

#include "device_common.cuh"

namespace malib {

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Stores v to the same place of CTA `rank` of the cluster, counting its 16 bytes on that
// CTA's mbarrier.
__device__ __forceinline__ void peer_store(void* dst, uint64_t* bar, uint32_t rank, float4 v) {
    asm volatile(
        "{\n .reg .b32 d, b;\n mapa.shared::cluster.u32 d, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
        " st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [d], {%3, %4, %5, %6}, [b];\n}" ::"r"(
            smem_u32(dst)),
        "r"(smem_u32(bar)), "r"(rank), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
        : "memory");
}

// mbar_wait_bounded for a barrier that peers complete: their stores are seen after it.
__device__ __forceinline__ bool peer_wait_bounded(uint64_t* bar, uint32_t parity, uint64_t limit_ns) {
    const uint64_t t0 = globaltimer_ns();
    while (true) {
        uint32_t ok;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
            " selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
        if (ok) return true;
        if (globaltimer_ns() - t0 > limit_ns) return false;
    }
}

}  // namespace malib
