// lla_plan.cuh -- what the kernels share that work out a batch's bookkeeping in one cluster (lla_pages.cu,
// lla_prefix_plan.cu): prefix sums over a CTA's threads, one thread per sequence, and the cluster's launch.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "lla_internal.h"

namespace lla {
namespace {

constexpr int kPlanThreads = 1024;  // a sequence each, too
static_assert(kPlanThreads == LLA_MAX_BATCH, "thread s plans sequence s");

// Exclusive prefix sums of two values over a CTA's threads, and the CTA's totals.  `part` has 33 entries.  Three barriers.
struct Two {
    unsigned long long a;
    int b;
};
__device__ __forceinline__ Two block_scan(Two v, Two *part, Two &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto scan = [&](Two x) {  // inclusive, of a warp
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long ua = __shfl_up_sync(0xffffffffu, x.a, o);
            const int ub = __shfl_up_sync(0xffffffffu, x.b, o);
            if (lane >= o) {
                x.a += ua;
                x.b += ub;
            }
        }
        return x;
    };
    const Two inc = scan(v);
    __syncthreads();  // part is free
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        const Two w = part[lane], all = scan(w);
        part[lane] = Two{all.a - w.a, all.b - w.b};
        if (lane == 31) part[32] = all;
    }
    __syncthreads();
    total = part[32];
    return Two{part[warp].a + inc.a - v.a, part[warp].b + inc.b - v.b};
}

// Clusters of more than 8 CTAs are an opt-in of the kernel, once per device.
template <typename K>
lla_status allow_clusters_of_16(K kern, DeviceOnce &once) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return LLA_ERR_CUDA;
    const bool cached = dev >= 0 && dev < 64;
    if (cached && once.done[dev].load(std::memory_order_acquire)) return LLA_OK;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return LLA_ERR_CUDA;
    if (cached) once.done[dev].store(true, std::memory_order_release);
    return LLA_OK;
}

// A cluster of `ctas` CTAs of kPlanThreads.
template <typename A>
lla_status launch_plan(void (*kern)(A), int ctas, const A &a, cudaStream_t stream, int smem = 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kPlanThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, a) == cudaSuccess ? LLA_OK : LLA_ERR_CUDA;
}

}  // namespace
}  // namespace lla
