// qmm_launch.cuh -- launches that may overlap the tail of the kernel before them (programmatic dependent launch), optionally in clusters.
#pragma once

#include <atomic>

#include "qmm_common.cuh"

namespace qmm {

template <typename... P, typename... A>
static qmm_status launch_pdl(void (*kern)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, const char* what, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cfg.attrs = attr;
    return check_cuda(cudaLaunchKernelEx(&cfg, kern, args...), what);
}

// Sets a kernel's attributes once per device: dynamic shared memory that may pass 48 KB together with static arrays, clusters of more than eight blocks.
// `configured`: one bit per device, a static of the caller's instantiation.
template <typename K> static qmm_status configure_once(std::atomic<uint64_t>& configured, K kern, size_t smem, bool wide_cluster, const char* what)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
    const uint64_t bit = dev < 64 ? (1ull << dev) : 0;
    if (configured.load(std::memory_order_relaxed) & bit) return QMM_OK;
    cudaError_t e = smem > 32 * 1024 ? cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) : cudaSuccess;
    if (e == cudaSuccess && wide_cluster) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return check_cuda(e, what);
    configured.fetch_or(bit, std::memory_order_relaxed);
    return QMM_OK;
}

}  // namespace qmm
