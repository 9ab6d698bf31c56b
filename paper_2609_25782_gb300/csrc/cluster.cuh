// Clusters of thread blocks: their barrier, their blocks' shared memory, and launches behind the kernel before
// (attend_kernels.cu, sparse_kernels.cu).
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace kvt {
namespace {

__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The kernel that comes next may be scheduled (it waits all the same for this one's end).
__device__ __forceinline__ void next_may_come() { asm volatile("griddepcontrol.launch_dependents;"); }

__device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// A launch as a programmatic dependent of the kernel before it on the stream: its blocks may be there when that one
// ends, and every thread waits for its end (after_previous) before it reads or writes anything. cluster > 0: each row
// of the grid, of `cluster` blocks, is a cluster.
template <typename... Args>
cudaError_t launch_behind(void (*kernel)(Args...), dim3 grid, int cluster, int threads, int smem, cudaStream_t st,
                          const Args &...args) {
    cudaLaunchConfig_t c{};
    cudaLaunchAttribute at[2];
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    c.attrs = at;
    c.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&c, kernel, args...);
}

// Prepares a kernel for clusters of up to 16 blocks and `most` bytes of shared memory, and tells how many clusters
// of 1, 2, 4, 8 and 16 blocks of `smem` bytes the device holds at once.
template <typename... Args>
cudaError_t fit_clusters(void (*kernel)(Args...), int threads, int most, int smem, int (&fit)[5]) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    for (int i = 0; i < 5 && e == cudaSuccess; ++i) {
        cudaLaunchConfig_t c{};
        cudaLaunchAttribute at[1];
        c.gridDim = dim3(1 << i);
        c.blockDim = dim3(threads);
        c.dynamicSmemBytes = smem;
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 1 << i;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        c.attrs = at;
        c.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&fit[i], kernel, &c);
    }
    return e;
}

}  // namespace
}  // namespace kvt
