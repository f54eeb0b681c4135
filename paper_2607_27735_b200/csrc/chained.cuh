// Launches of small kernels that may begin under the end of the kernel before them.
#pragma once

#include "spec_common.cuh"

namespace spec {

// First thing in a kernel that launch_chained starts: waits for the results of the kernel before it.  The next kernel is
// let go only after that wait, so whatever starts early under this kernel finds everything before it complete.  What an earlier
// kernel may have written is read by ordinary loads, never through the read-only path, which the compiler could move
// ahead of the wait.
__device__ __forceinline__ void stream_wait()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// The same for a kernel whose results later kernels read through the read-only path (page tables): nothing starts under it,
// so no SM holds lines of them from before.
__device__ __forceinline__ void stream_wait_only() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// cluster > 1: that many neighbouring CTAs along x form a cluster.
template <typename... P, typename... A>
int launch_chained(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kern, args...) != cudaSuccess) {
        cudaGetLastError();
        return SPEC_ERR_CUDA;
    }
    count_launch(1);
    return SPEC_OK;
}

}  // namespace spec
