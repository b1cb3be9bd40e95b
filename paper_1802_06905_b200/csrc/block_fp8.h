// The 8-bit product as a sequence of launches.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/cconv_block.h"

namespace cconv {

int64_t fp8_workspace(const cconv_fp8_product_args& a, int sms);
// Sizes are positive, operands checked.  A status code.
int run_fp8(const cconv_fp8_product_args& a, int sms, cudaStream_t s);

}  // namespace cconv
