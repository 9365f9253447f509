// Host side shared by the translation units of libef21: error returns, sizes and the launch of a kernel.
#pragma once
#include "../../include/ef21.h"

#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>
#include <set>
#include <utility>

#include "common.cuh"

#define CU(call)                                         \
    do {                                                 \
        cudaError_t e__ = (call);                        \
        if (e__ != cudaSuccess) return EF21_ERR_CUDA;    \
    } while (0)
#define EF(call)                                         \
    do {                                                 \
        ef21_status s__ = (call);                        \
        if (s__ != EF21_OK) return s__;                  \
    } while (0)

namespace ef21 {

constexpr size_t ALIGN = 256;
inline size_t align_up(size_t v) { return (v + ALIGN - 1) / ALIGN * ALIGN; }
inline i64 ceil_div(i64 a, i64 b) { return (a + b - 1) / b; }

// Kernel launch as a programmatic dependent of whatever precedes it in the stream (see pdl_wait), with clusters of C blocks.
template <typename... Params, typename... Args>
cudaError_t launch(void (*kern)(Params...), dim3 grid, unsigned block, size_t smem, cudaStream_t st, unsigned C, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = C; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = C > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<Params>(args)...);
}

// Opt-in of a kernel to more dynamic shared memory than the default 48 KB (and to clusters of more than eight blocks): an
// attribute per device, set once.
inline ef21_status allow_smem(const void* kern, size_t bytes, bool big_cluster = false) {
    static std::mutex mu;
    static std::set<std::pair<int, const void*>> done;
    int dev = -1;
    CU(cudaGetDevice(&dev));
    std::lock_guard<std::mutex> lock(mu);
    if (done.count({dev, kern})) return EF21_OK;
    CU(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    if (big_cluster) CU(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    done.insert({dev, kern});
    return EF21_OK;
}

}  // namespace ef21
