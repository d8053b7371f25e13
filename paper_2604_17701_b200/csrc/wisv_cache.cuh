// What the files behind wisv_cache share: the context, checks and the launch.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/wisv.h"
#include "wisv_attn.cuh"

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct wisv_cache {
    wisv_cache_config cfg;
    int device = 0;
    int sm_count = 0;
    int page_shift = 0;
    int64_t launches = 0;
    // one allocation: [error word, half of the counters in use | arrival counters | partial maxima and sums | partial outputs]
    void* work = nullptr;         // NULL: the caller's
    int32_t* err = nullptr;
    int32_t* count = nullptr;
    float2* part_ml = nullptr;
    float* part_o = nullptr;
    EncodeTiledFn encode = nullptr;
    uint64_t wait_clocks = wisv::kAttnWaitClocks;       // wisv_debug_cache_waits
    int32_t stalled = -1;
};

namespace wisv {

// Shared-memory limits of the kernels of wisv_q8.cu on the current device.
bool q8_prepare();

namespace {

#define WISV_TRY_CUDA(call)                                                        \
    do {                                                                           \
        if ((call) != cudaSuccess) { (void)cudaGetLastError(); return WISV_ECUDA; } \
    } while (0)

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline int log2_exact(int x)
{
    for (int s = 0; s < 31; ++s) if ((1 << s) == x) return s;
    return -1;
}

// One kernel on `st`, as a cluster of `cluster` blocks when that is more than 1, with programmatic dependent launch: its blocks are
// set up while the kernel before it in the stream ends, and wait for it (griddepcontrol.wait) before they read anything.
template <typename P>
int launch(void (*kernel)(P), int grid, int block, size_t smem, int cluster, cudaStream_t st, const P& p)
{
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    WISV_TRY_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
    return WISV_OK;
}

// A cache's workspace and launch shapes are those of the device that it was created on.
inline int check_device(const wisv_cache* c)
{
    int dev = 0;
    WISV_TRY_CUDA(cudaGetDevice(&dev));
    return dev == c->device ? WISV_OK : WISV_EINVAL;
}

}  // namespace

}  // namespace wisv
