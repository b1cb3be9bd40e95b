// The block quantiser's parameters and launcher.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace cconv {

struct QuantParams {
  int64_t T, D;
  const void* x;
  uint8_t* q;
  float* scale;
  int64_t x_rs, x_cs, q_rs, q_cs, scale_rs, scale_cs;
  int64_t row_blocks;  // filled in by the launcher
};

cudaError_t run_quantize(const QuantParams& p, int dtype, int block_rows, int sms, cudaStream_t s);

}  // namespace cconv
