// Products of a few tokens: weights stream through registers once.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "block.h"

namespace cconv {

constexpr int64_t kFewTokens = 16, kFewTokensInParts = 4;

// Whether rows x k weights (es bytes an element) and tokens can be read by these kernels: k contiguous in
// pieces of 16 bytes, addresses and pitches multiples of 16 bytes.
bool few_readable(const Mat& m, int64_t rows, int64_t k, int es);

// h[t][f] = act(x[t] . wg[f]) * (x[t] . wu[f]), T <= kFewTokens; the dot products too, if asked for, and, if
// h_lo (which lies like h) is there, what the rounding of h to the type left, rounded itself.
cudaError_t run_few_gated(const Mat& x, const Mat& wg, const Mat& wu, const Mat& gate_pre, const Mat& up_pre,
                          const Mat& h, const Mat& h_lo, int64_t T, int64_t F, int64_t D, int act, int dtype, int sms,
                          cudaStream_t s);
// out[t][n] = (x[t] + x_lo[t]) . w[n]; x_lo lies like x, or is absent (T > kFewTokensInParts).  weights_there: run_few_gated of the same call is in front, which does not write w.
cudaError_t run_few_product(const Mat& x, const Mat& x_lo, const Mat& w, const Mat& out, int64_t T, int64_t N,
                            int64_t K, int dtype, int sms, bool weights_there, cudaStream_t s);
// out[t][n] = sum_kb sa[t][kb] sb[n/128][kb] (x[t] . w[n])_kb of 8-bit x and w.
cudaError_t run_few_fp8(const Mat& x, const Mat& w, const Mat& sa, const Mat& sb, const Mat& out, int64_t T, int64_t N,
                        int64_t K, int dtype, int sms, cudaStream_t s);

}  // namespace cconv
