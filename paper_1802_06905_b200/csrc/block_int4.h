// Products with 4-bit weights, and their quantiser.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "block.h"

namespace cconv {

int64_t int4_workspace(const cconv_int4_product_args& a, int sms);
int run_int4(const cconv_int4_product_args& a, int sms, cudaStream_t s);  // M, N, K > 0
cudaError_t run_quantize_groups(const cconv_quantize_groups_args& a, cudaStream_t s);

}  // namespace cconv
