// Blocks of one thread-block cluster: barrier, and reads of one another's shared memory.
#pragma once
#include "common.cuh"

namespace ef21 {

__device__ __forceinline__ unsigned cluster_rank() {
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned cluster_blocks() {
    unsigned n;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}
// All threads of all blocks; what they wrote to shared memory is visible behind it.
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// The address, in the cluster's shared memory, of block `rank`'s copy of a variable.
__device__ __forceinline__ unsigned remote_address(const void* mine, unsigned rank) {
    unsigned at = (unsigned)__cvta_generic_to_shared(mine), remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(at), "r"(rank));
    return remote;
}
__device__ __forceinline__ double remote_double(const double* mine, unsigned rank) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(remote_address(mine, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float remote_float(const float* mine, unsigned rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote_address(mine, rank)) : "memory");
    return v;
}
// Sums over the blocks of the cluster, in their order, in thread 0 of rank 0; v counts in thread 0 of every block.  mine: N doubles of shared memory.
template <int N>
__device__ __forceinline__ void cluster_sums(double (&v)[N], double* mine) {
    const unsigned C = cluster_blocks();
    if (C == 1) return;
    if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) mine[k] = v[k];
    }
    cluster_barrier();
    if (cluster_rank() == 0 && threadIdx.x == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.0;
            for (unsigned r = 0; r < C; ++r) v[k] += remote_double(mine + k, r);
        }
    }
    cluster_barrier();                                       // nobody leaves while it is read
}

}  // namespace ef21
