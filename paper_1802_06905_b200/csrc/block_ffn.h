// The gated feed-forward block as a sequence of launches.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/cconv_block.h"

namespace cconv {

// Bytes of workspace of a call on a device of `sms` SMs.
int64_t ffn_workspace(const cconv_ffn_args& a, bool backward, int sms);
// Launches the call; sizes are positive, operands checked.  A status code.
int run_ffn(const cconv_ffn_args& a, bool backward, int sms, cudaStream_t s);

}  // namespace cconv
