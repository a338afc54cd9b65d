// Chains of short kernels on one stream: each may be set up while the one before it still runs (programmatic stream
// serialisation), and waits for that one's end before it touches memory.
#pragma once
#include "mw_common.cuh"

namespace mw {

// Every thread of a kernel launched by launch_after calls this first, before it reads or writes global memory: the
// kernels before are complete afterwards, and what they wrote is visible.  The next kernel of the chain may be set
// up from here on.
__device__ __forceinline__ void after_previous() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <typename... Params, typename... Args>
inline mw_status launch_after(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ++g_launch_count;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
}

}  // namespace mw
