// Launch of a kernel that may be set up while the one before it in the stream finishes; the kernel itself waits for
// that one (griddepcontrol.wait) before it reads or writes anything.
#pragma once

#include <algorithm>
#include <utility>

#include "remp_internal.h"

namespace remp {

#ifdef __CUDACC__
// First thing in such a kernel: the one before it has to be complete, and what it has written is visible then. Kernels that write
// caches, tables or counts stop here: the next kernel is set up when they are done.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Kernels that only read those let the next one be set up now.
__device__ __forceinline__ void grid_begin() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    grid_wait();
}
#endif

// In clusters of `cluster` thread blocks (at most 8; 1: none).
template <class... KArgs, class... Args>
cudaError_t launch_after_in_clusters(void (*kernel)(KArgs...), int64_t grid, int cluster, int threads, size_t smem, cudaStream_t stream, Args&&... args) {
    if (smem > 48 * 1024) {
        // once for each kernel and device: the attribute stays with the function
        static thread_local std::vector<std::pair<void*, int>> set;
        int device = -1;
        if (cudaError_t e = cudaGetDevice(&device)) return e;
        const std::pair<void*, int> key(reinterpret_cast<void*>(kernel), device);
        bool known = false;
        for (const auto& k : set) known |= k == key;
        if (!known) {
            if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, std::max(227 * 1024 - 4096, (int)smem))) return e;
            set.push_back(key);
        }
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid, 1, 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...)) return e;
    count_launch();
    return cudaGetLastError();
}

template <class... KArgs, class... Args>
cudaError_t launch_after(void (*kernel)(KArgs...), int64_t grid, int threads, size_t smem, cudaStream_t stream, Args&&... args) {
    return launch_after_in_clusters(kernel, grid, 1, threads, smem, stream, std::forward<Args>(args)...);
}

}  // namespace remp
