// Products of a few tokens: weights stream through registers once.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "block.h"

namespace cconv {

constexpr int64_t kFewTokens = 8;

// Whether rows x k weights (es bytes an element) and tokens can be read by these kernels: k contiguous in
// pieces of 16 bytes, addresses and pitches multiples of 16 bytes.
bool few_readable(const Mat& m, int64_t rows, int64_t k, int es);

// h[t][f] = act(x[t] . wg[f]) * (x[t] . wu[f]), T <= kFewTokens; the dot products too, if asked for.
// chained: may start while the kernel in front of it in the same call ends; more: another one follows.
cudaError_t run_few_gated(const Mat& x, const Mat& wg, const Mat& wu, const Mat& gate_pre, const Mat& up_pre,
                          const Mat& h, int64_t T, int64_t F, int64_t D, int act, int dtype, int sms, bool more,
                          cudaStream_t s);
// out[t][n] = x[t] . w[n]; w was there before the call that this launch belongs to.
cudaError_t run_few_product(const Mat& x, const Mat& w, const Mat& out, int64_t T, int64_t N, int64_t K, int dtype,
                            int sms, bool chained, bool more, cudaStream_t s);
// out[t][n] = sum_kb sa[t][kb] sb[n/128][kb] (x[t] . w[n])_kb of 8-bit x and w.
cudaError_t run_few_fp8(const Mat& x, const Mat& w, const Mat& sa, const Mat& sb, const Mat& out, int64_t T, int64_t N,
                        int64_t K, int dtype, int sms, cudaStream_t s);

}  // namespace cconv
