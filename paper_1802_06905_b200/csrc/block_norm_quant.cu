// Residual norms with 8-bit results: the forward kernels of block_norm_forward.cuh, whose last step gives
//
//   x = r' rho_r w_pre,  scale = max|x| / 448 over 128 channels of a token,  q = e4m3(x / scale)
//
// x stays in registers between the norm's sum, the maximum and the rounding, so that a token's channels pass
// through memory once: r and y are read, r' and q written.  x is not rounded to 16 bits in between (as two calls,
// residual_norm_forward and quantize_blocks, would).
#include "block_norm_forward.cuh"

namespace cconv {

cudaError_t run_norm_quantize(const NormParams& p, int dtype, int sms, cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16) return launch_forward<__nv_bfloat16, true>(p, sms, s);
  if (dtype == CCONV_TYPE_FP16) return launch_forward<__half, true>(p, sms, s);
  return launch_forward<float, true>(p, sms, s);
}

}  // namespace cconv
