// Programmatic dependent launch: a kernel of a call starts while the call's
// previous one still runs, sets itself up, and waits for it before it touches
// what that kernel writes.  The first kernel of a call is launched plainly, so
// nothing of a call starts before the stream's earlier work is done.
#pragma once

#include <cuda_runtime.h>

namespace flare {

// Lets the call's next kernel be launched once every CTA got here.
__device__ __forceinline__ void pdl_launch_next() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Waits until the call's previous kernel has completed and its writes are
// visible.  On every path out of the kernel: one that ended without it could
// let the stream's next work start beside the previous kernel.
__device__ __forceinline__ void pdl_wait() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Launches `kernel` behind the previous kernel of the stream with that
// overlap (`after`), in clusters of `cluster` CTAs.
template <typename... P, typename... A>
inline cudaError_t pdl_launch(void (*kernel)(P...), dim3 grid, int threads, int smem,
                              cudaStream_t stream, bool after, int cluster, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (after) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace flare
