// Launching a kernel while the one in front of it on the stream still runs.
#pragma once
#include <cuda_runtime.h>

namespace speca {
namespace {

// The kernel may begin as soon as all blocks of the one in front have (or have ended); it sets itself up, then waits here for all that that one does.
// Nothing in memory is touched before. A kernel in front that is not of this kind ends first, as ever. (Without this, single products
// of a loop began on ticks of 2.05 us: 4 rows x 6144 x 4096 10.3 us a call, 8.2 with it; 4096 x 4608 x 1152 with GELU into 8 bits 30.7, 28.4.)
__device__ __forceinline__ void wait_for_stream() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), unsigned blocks, unsigned cluster, unsigned threads, unsigned smem, cudaStream_t stream,
                         const Args&... args) {
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(blocks);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&config, kernel, static_cast<Params>(args)...);
}

}  // namespace
}  // namespace speca
