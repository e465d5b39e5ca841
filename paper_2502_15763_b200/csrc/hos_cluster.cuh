// Blocks of a cluster: who is who, their barrier, and writing to one another's shared memory.
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
// The same, where a cluster may be a single block: the block's own barrier then (30 cycles instead of 900).
__device__ __forceinline__ void cluster_or_block_sync() {
    if (cluster_size() == 1) __syncthreads();
    else cluster_sync();
}
// "All blocks have begun", for the first write to another's shared memory, in two halves with work of one's own in between.  Orders no
// memory: with the fence of a release the first half took 1.2 us.
__device__ __forceinline__ void cluster_begun_arrive() {
    if (cluster_size() > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_begun_wait() {
    if (cluster_size() > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
// Writes to another block's shared memory, where *mine is in this one's.  That block must have begun (a barrier of the cluster before)
// and sees it after the next barrier.
__device__ __forceinline__ uint32_t address_in_block(const void* mine, int block) {
    uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(mine));
    asm("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(a) : "r"(block));
    return a;
}
__device__ __forceinline__ void write_to_block(double* mine, int block, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" :: "r"(address_in_block(mine, block)), "d"(v) : "memory");
}
__device__ __forceinline__ void write_to_block(int4* mine, int block, const int4& v) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(address_in_block(mine, block)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}

}  // namespace hos
