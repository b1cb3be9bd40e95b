// Kernel launches of the feed-forward sub-block.
#pragma once
#include <cuda_runtime.h>

namespace cconv {
namespace {

// An ordinary launch, or one that may start while the kernel in front of it (of the same call) ends; all
// kernels here wait for that kernel before they touch memory.
template <typename F, typename... Args>
cudaError_t launch(F f, dim3 grid, int threads, size_t smem, int cluster, bool chained, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (chained) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = unsigned(cluster);
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = unsigned(n);
  return cudaLaunchKernelEx(&cfg, f, args...);
}

}  // namespace
}  // namespace cconv
