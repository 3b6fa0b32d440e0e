// Host-side helpers shared by the entry points: the caller's current device, programmatic dependent launches.
#pragma once
#include <cuda_runtime.h>

#include <utility>

namespace ftmoe {

// Restores the calling thread's current device when the entry point returns.
struct DeviceScope {
  int prev = -1;
  cudaError_t err;
  explicit DeviceScope(int dev) {
    err = cudaGetDevice(&prev);
    if (err == cudaSuccess && prev != dev) err = cudaSetDevice(dev); else prev = -1;
  }
  ~DeviceScope() { if (prev >= 0) (void)cudaSetDevice(prev); }
};

// A launch the stream's next kernel may be scheduled beside: every kernel launched this way waits for all before it (grid_wait)
// before it touches memory that a kernel or a copy of the stream writes, so only launch latency and prologues overlap.
// cluster > 1: blocks in clusters of that many.
template <typename... P, typename... Args>
cudaError_t launch_clusters(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, Args &&...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

template <typename... P, typename... Args>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, Args &&...args) {
  return launch_clusters(kernel, grid, threads, smem, 1, st, std::forward<Args>(args)...);
}

}  // namespace ftmoe
