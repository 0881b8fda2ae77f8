// Barrier and shared memory of a thread-block cluster.
#pragma once

#include <stdint.h>

namespace mbscan {

// Every thread of the cluster arrives, then waits; what was written before is visible after.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// *p as it is in the shared memory of CTA `cta` of the cluster, which must not have ended.
__device__ __forceinline__ uint32_t cluster_address(const void *p, int cta) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(cta));
    return r;
}
__device__ __forceinline__ int cluster_load(const int *p, int cta) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(cluster_address(p, cta)) : "memory");
    return v;
}
__device__ __forceinline__ float cluster_load(const float *p, int cta) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_address(p, cta)) : "memory");
    return v;
}

}  // namespace mbscan
