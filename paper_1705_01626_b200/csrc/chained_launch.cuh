// Launches that may begin before the kernel in front of them on the stream has ended (programmatic dependent launch).
// Such a kernel sets itself up, then waits for all work in front of it -- let_next_start() and wait_for_previous()
// are the two ends -- before it touches any memory of the caller.  A kernel that cannot begin early simply finds
// nothing to wait for.  As it may have begun before its inputs were written, it must not read them through the
// read-only path (ld.global.nc, __ldg).  It hides the start of a kernel of a few microseconds behind the end of the one before.
#pragma once

#include <cuda_runtime.h>

#include "zvc_common.cuh"

namespace cdma {

__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The same in front of bulk copies: they read memory by another way than the stores of the kernel in front went, and the
// fence orders the two.
__device__ __forceinline__ void wait_before_copies() {
    wait_for_previous();
    asm volatile("fence.proxy.async.global;" ::: "memory");
}
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// cluster: CTAs per cluster, 0 where the kernel has that fixed or has none.
template <typename... Params, typename... Args>
cudaError_t launch_chained(void (*kernel)(Params...), uint32_t grid, uint32_t threads, uint32_t smem, uint32_t cluster,
                           cudaStream_t stream, const Args&... args) {
    cudaLaunchAttribute attributes[2] = {};
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim = {cluster, 1, 1};
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(grid);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = attributes;
    config.numAttrs = cluster != 0 ? 2 : 1;
    count_kernel_launch();
    return cudaLaunchKernelEx(&config, kernel, args...);
}

}  // namespace cdma
