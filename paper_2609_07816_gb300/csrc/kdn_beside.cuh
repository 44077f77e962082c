// kdn_beside.cuh -- kernels of one call that overlap.
//
// A kernel's CTAs say with let_next_start that the next kernel of the stream may start
// once all of them have said so (its CTAs take the room that falls free).  The next one is
// launched with launch_beside and either
//   waits, before it reads what the first one writes (wait_for_previous), or
//   needs nothing of it and only ends after it (end_after_previous, by one CTA), so that
//   what follows in the stream comes after both.
#pragma once

#include "kdn_internal.cuh"

namespace kdn {

__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void end_after_previous() {
  if (threadIdx.x == 0 && blockIdx.x + 1 == gridDim.x && blockIdx.y + 1 == gridDim.y && blockIdx.z + 1 == gridDim.z)
    wait_for_previous();
}

template <typename... P, typename... A>
kdn_status_t launch_beside(void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t s, const A &...args) {
  cudaLaunchAttribute beside{};
  beside.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  beside.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = grid;
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = smem;
  c.stream = s;
  c.attrs = &beside;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, args...) == cudaSuccess ? KDN_OK : KDN_ERR_CUDA;
}

}  // namespace kdn
