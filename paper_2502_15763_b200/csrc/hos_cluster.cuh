// Blocks of a cluster: who is who, their barrier, and reading one another's shared memory.
#pragma once

#include <stdint.h>

namespace hos {

__device__ __forceinline__ int cluster_rank() {
    int r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ int cluster_size() {
    int r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// Barrier of all threads of the cluster; what was written before it, to global memory and to shared, is seen after it.
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The 64-bit word of another block's shared memory that lies where *mine does in this one's.
__device__ __forceinline__ unsigned long long read_of_block(const void* mine, int block) {
    uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(mine));
    unsigned long long v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(block));
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}

}  // namespace hos
