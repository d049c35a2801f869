// Kernel launches with programmatic stream serialisation and clusters, from the host.
#pragma once

#include <cuda_runtime.h>
#include <string.h>

#include "../../include/adasd.h"

#define CUDA_TRY(expr)                         \
    do {                                       \
        cudaError_t e__ = (expr);              \
        if (e__ != cudaSuccess) return ADASD_ERR_CUDA; \
    } while (0)

namespace adasd {

// early: launch with programmatic stream serialisation: the kernel may become resident while the one ahead of
// it is still running (it waits before it reads what that one wrote).  cs: CTAs per cluster; 0: the kernel
// uses no cluster.  (A kernel that uses cluster-scope instructions gets the attribute even for clusters of one.)
template <typename K, typename... Args>
int launch_kernel(bool early, K kernel, int grid, int threads, int smem, int cs, cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3((unsigned)grid, 1, 1);
    lc.blockDim = dim3((unsigned)threads, 1, 1);
    lc.dynamicSmemBytes = (size_t)smem;
    lc.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = early ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cs;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = cs > 0 ? 2 : 1;
    CUDA_TRY(cudaLaunchKernelEx(&lc, kernel, args...));
    return ADASD_OK;
}
template <typename K, typename... Args>
int launch_pdl(K kernel, int grid, int threads, int smem, int cs, cudaStream_t stream, const Args&... args) {
    return launch_kernel(true, kernel, grid, threads, smem, cs, stream, args...);
}

}  // namespace adasd
