// jb_launch.cuh -- launches whose start overlaps the end of the kernel before them.
#pragma once
#include <cuda_runtime.h>

namespace jb {

// Waits until the kernels before this one are done and what they wrote is visible. Every thread of a
// kernel that launch() starts calls it before it touches memory.
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Lets the next kernel's CTAs start; they wait in after_previous() until this kernel is done.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Enqueues a kernel on clusters of `cluster` CTAs (0: none).
template <typename... Params, typename... Args>
cudaError_t launch(void (*kernel)(Params...), dim3 grid, unsigned block, size_t shared, unsigned cluster, cudaStream_t s,
                   const Args&... args) {
    cudaLaunchAttribute a[2];
    a[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a[0].val.programmaticStreamSerializationAllowed = 1;
    a[1].id = cudaLaunchAttributeClusterDimension;
    a[1].val.clusterDim.x = cluster;
    a[1].val.clusterDim.y = a[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = dim3(block);
    c.dynamicSmemBytes = shared;
    c.stream = s;
    c.attrs = a;
    c.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&c, kernel, static_cast<Params>(args)...);
}

}  // namespace jb
