// Kernel launches of the feed-forward sub-block.
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

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

// Lets a kernel have `bytes` of dynamic shared memory on the current device (`ready`: the kernel's, by device).
template <typename F>
cudaError_t allow_smem(F f, bool (&ready)[64], int bytes) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!__atomic_load_n(&ready[dev & 63], __ATOMIC_ACQUIRE)) {
    e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    __atomic_store_n(&ready[dev & 63], true, __ATOMIC_RELEASE);
  }
  return cudaSuccess;
}

// How many clusters of `size` (2 to 8) blocks of f the current device holds at once (`known`: the kernel's, by device and size,
// one more than the number).
template <typename F>
cudaError_t clusters_at_once(F f, int threads, int smem, int size, std::atomic<int> (&known)[64][9], int* n) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  std::atomic<int>& at = known[dev & 63][size];
  *n = at.load(std::memory_order_relaxed) - 1;
  if (*n >= 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(size));
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = size_t(smem);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(size);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(n, f, &cfg);
  if (e == cudaSuccess) at.store(*n + 1, std::memory_order_relaxed);
  return e;
}

// Shared memory to ask for, at least `need`, so that no SM takes more than its share of `blocks`: what is left is filled
// up before other SMs get any (256 blocks of which three fit an SM may lie on 86 of them).
constexpr int kSpreadSmem = 115 * 1024;  // at most
inline int spread_smem(int64_t blocks, int sms, int need) {
  const int64_t each = std::max<int64_t>(1, cdiv64(blocks, sms));
  // (an SM has 228 KB, 1 KB a block of it for itself)
  return std::max(need, int(228 / (each + 1)) * 1024);
}

}  // namespace
}  // namespace cconv
