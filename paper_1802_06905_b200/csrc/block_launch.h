// Kernel launches of the feed-forward sub-block.
#pragma once
#include <cuda_runtime.h>

#include "block.h"

namespace cconv {
namespace {

// Launches f so that it may start while the kernel in front of it on the stream ends (start_in_order() in
// the kernel keeps the order of memory).
template <typename F, typename... Args>
cudaError_t launch(F f, dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(cluster);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, f, args...);
  block_launches() += e == cudaSuccess;
  return e;
}

}  // namespace
}  // namespace cconv
