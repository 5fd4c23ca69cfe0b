// Clusters: rank, barrier, stores to a peer's shared memory and loads from it. Only for
// launches with a cluster dimension: without one these are illegal instructions.
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

// Writes 8 or 16 bytes to the same place of CTA `rank` of the cluster, seen after the next cluster barrier.
__device__ __forceinline__ void peer_put(float2* dst, uint32_t rank, float2 v) {
    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %0, %1;\n st.shared::cluster.v2.f32 [a], {%2, %3};\n}" ::"r"(
                     smem_u32(dst)),
                 "r"(rank), "f"(v.x), "f"(v.y)
                 : "memory");
}

__device__ __forceinline__ void peer_put(float4* dst, uint32_t rank, float4 v) {
    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %0, %1;\n st.shared::cluster.v4.f32 [a], {%2, %3, %4, %5};\n}" ::"r"(
                     smem_u32(dst)),
                 "r"(rank), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
                 : "memory");
}

// Reads the same place of CTA `rank` of the cluster, after a cluster barrier that follows its writes.
__device__ __forceinline__ uint64_t peer_load(const uint64_t* src, uint32_t rank) {
    uint64_t v;
    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %1, %2;\n ld.shared::cluster.u64 %0, [a];\n}"
                 : "=l"(v)
                 : "r"(smem_u32(src)), "r"(rank)
                 : "memory");
    return v;
}
__device__ __forceinline__ uint32_t peer_load(const uint32_t* src, uint32_t rank) {
    uint32_t v;
    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %1, %2;\n ld.shared::cluster.u32 %0, [a];\n}"
                 : "=r"(v)
                 : "r"(smem_u32(src)), "r"(rank)
                 : "memory");
    return v;
}
__device__ __forceinline__ float4 peer_load(const float4* src, uint32_t rank) {
    float4 v;
    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %4, %5;\n ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n}"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(smem_u32(src)), "r"(rank)
                 : "memory");
    return v;
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
