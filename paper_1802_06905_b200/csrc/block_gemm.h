// Products of the feed-forward block: parameters and launchers.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "block.h"

namespace cconv {

// C32[m][n] (+)= sum_k A[m][k] B[n][k], fp32, row-major, pitch N.
cudaError_t run_product_simple(const Mat& a, const Mat& b, float* c, int64_t M, int64_t N, int64_t K, int dtype,
                               bool add, cudaStream_t s);
// 8-bit operands with their scales.
cudaError_t run_fp8_simple(const Mat& a, const Mat& b, const Mat& sa, const Mat& sb, const Mat& c, int64_t M,
                           int64_t N, int64_t K, int dtype, cudaStream_t s);

// What becomes of finished sums [M][N] in fp32.
cudaError_t finish_store(const float* sums, const Mat& out, int64_t M, int64_t N, int dtype, cudaStream_t s);
cudaError_t finish_gated(const float* g, const float* u, const Mat& gate_pre, const Mat& up_pre, const Mat& h,
                         int64_t M, int64_t N, int act, int dtype, cudaStream_t s);
cudaError_t finish_gated_backward(const float* dh, const Mat& gate_pre, const Mat& up_pre, const Mat& dg,
                                  const Mat& du, const Mat& h, int64_t M, int64_t N, int act, int dtype,
                                  cudaStream_t s);

}  // namespace cconv
