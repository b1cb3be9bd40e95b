// A mixture-of-experts layer for a few tokens: launches.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "block.h"

namespace cconv {

constexpr int64_t kMostExperts = 1024, kMostChosen = 32;

int64_t moe_workspace(const cconv_moe_args& a, int sms);
int run_moe(const cconv_moe_args& a, int sms, cudaStream_t s);  // T, D, E > 0; F = 0: the router alone

}  // namespace cconv
