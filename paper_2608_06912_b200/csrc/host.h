// Host helpers shared by the library's translation units: launch counting, the thread's last CUDA error, and the
// launch itself (programmatic stream serialisation, see pdl_wait in common.cuh).
#pragma once
#include <cuda_runtime.h>

#include "../../include/lapsum.h"

namespace lapsum {

int cuda_fail(cudaError_t e);  // remembers e for lapsum_last_cuda_error, returns LAPSUM_ERR_CUDA
int post_launch();             // counts a launch and picks up its error

template <typename... KArgs, typename... Args>
int launch_clusters(unsigned cluster, void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t st, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
    return e != cudaSuccess ? cuda_fail(e) : post_launch();
}

template <typename... KArgs, typename... Args>
int launch_pdl(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t st, const Args &...args)
{
    return launch_clusters(1, kernel, grid, block, smem, st, args...);
}

}  // namespace lapsum
