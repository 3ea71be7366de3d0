// Launches of one call's kernels in a chain: each may be scheduled while its predecessor drains (programmatic dependent
// launch) and waits for the predecessor's results itself.
//
// Every kernel of a chain calls chain_next() (its successor may be scheduled) and chain_wait() before it touches memory that
// others write or read: chain_wait returns once the predecessor has finished, which had waited for its own predecessor.
// In every CTA some thread waits, also in one without work: a grid of which none had could end before its predecessor, and what
// follows the call on its stream waits for the last grid alone.
// The first kernel of a call is launched with `first`, an ordinary launch behind whatever the stream holds.
#pragma once

#include <utility>

#include "cast_internal.h"

namespace cast {

__device__ __forceinline__ void chain_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void chain_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <class... P, class... A>
int launch_chained(bool first, void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t stream, int cluster, A&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    unsigned n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)cluster;
        attr[n].val.clusterDim.y = 1;
        attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (!first) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    CAST_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, P(std::forward<A>(args))...));
    count_launch();
    return CAST_OK;
}

}  // namespace cast
