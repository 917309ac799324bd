// fw_chain.cuh -- kernels that start while the one before them on the stream ends.
//
// A kernel launched by launch_chained() may find its CTAs on the GPU as soon as all CTAs of the kernel before have started
// and said so (or left), whoever's it is; it sets up what needs no memory, and waits for that kernel's end, and so for
// all before it, in wait_for_the_one_before().  Every thread calls that before it reads or writes global memory, and no thread
// leaves without: a kernel that ended without having waited would let the next one pass its own wait too soon.  One kernel reads
// before its wait, k_pages_fork_end: tables that the kernel before it, k_pages_fork, does not change, and that all kernels before
// that one are done with, since it lets the next start only behind its own wait.  A decode step's rotation, append and attention
// in a graph: 8 cells of 512 rows 13.2 us (14.3 launched one after another), of 4,096 17.1 (18.2), 64 of 1,024 20.3 (21.3).
#pragma once

#include "fw_internal.h"

namespace fw {

__device__ __forceinline__ void wait_for_the_one_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_the_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// cluster: CTAs of a cluster along x, 0: none.
template <typename... P, typename... A>
fw_status launch_chained(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, const A &...args)
{
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = cluster ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? FW_OK : FW_ERR_CUDA;
}

}  // namespace fw
