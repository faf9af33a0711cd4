// Kernels that follow one another on a stream, with the launch of the next hidden behind the end of the last.
//
// A kernel launched through launch_chained may be set up, and its blocks made resident, while its predecessor on the stream
// still runs; it must begin with wait_for_predecessor(), in every thread, before it touches memory: that returns when the
// predecessor has completed and what it wrote is visible.  Since no thread of such a kernel ends before that, its own
// successor may in turn rely on everything before it.  let_successor_in() only permits the early set-up (it takes
// effect once every block of the grid has said it or ended); a successor that was launched the ordinary way ignores it.
//
// Such a kernel's pointer parameters are not __restrict__, and it uses no non-coherent loads: both promise that nobody else
// writes the data while the kernel runs, which begins here while the predecessor still writes, and would let the compiler
// move a load in front of the wait.
#pragma once

#include <cuda_runtime.h>

#include <utility>

namespace dpk {

__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_successor_in() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... P, typename... A>
static cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
  if (e != cudaSuccess) cudaGetLastError();      // reported to the caller here, not to whoever asks next
  return e;
}

// The same in clusters of two blocks (2 * pairs blocks).
struct Pairs { unsigned n; };
template <typename... P, typename... A>
static cudaError_t launch_chained(void (*kernel)(P...), Pairs pairs, dim3 block, size_t smem, cudaStream_t s, A&&... args) {
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * pairs.n);
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}

}  // namespace dpk
