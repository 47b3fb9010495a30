// Launches whose start may overlap the end of the kernel before them in the stream (programmatic dependent launch).
//
// A kernel launched this way calls overlap_begin() once, which lets the next such kernel start when every CTA has done so
// and as SMs have room; it does what needs no global memory, and calls overlap_wait() in EVERY thread that touches global memory, before it does:
// the call returns when the kernels before it in the stream have finished and their writes are visible.  Its loads are ordinary
// ones: the read-only path (__ldg) asks for data that stays as it is for the kernel's whole life.  Kernels launched in
// the ordinary way, before or after, are not affected.  What is gained is the launch latency and the set-up of the
// next kernel: 1 to 1.5 us of each call in a row of small ones (one row, inner 256, 1536 features: 4.4 -> 3.1 us).
#pragma once

#include <cuda_runtime.h>

namespace sdvg {

__device__ __forceinline__ void overlap_begin() { cudaTriggerProgrammaticLaunchCompletion(); }
__device__ __forceinline__ void overlap_wait() { cudaGridDependencySynchronize(); }

// cluster: CTAs per cluster where the kernel does not fix it itself, else 0.
template <class Params>
cudaError_t launch_overlapped(void (*kernel)(Params), unsigned grid, int threads, size_t dynamic_bytes, int cluster,
                              cudaStream_t stream, const Params& params) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = dynamic_bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 0 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, params);
  if (e != cudaSuccess) cudaGetLastError();            // reported here; the next call must not find it again
  return e;
}

}  // namespace sdvg
