// The 8-bit product with a scale for each block of 128, as a sequence of launches.
//
// C[m][n] = sum_kb sa[m][kb] sb[n/128][kb] (A B^T)_kb: the tensor cores form the sums of one block of 128
// (one stage: 128 bytes of k a row), which the epilogue warps scale and add up in fp32 registers while the
// next block's are formed.  Up to 16 tokens go through the kernel that streams the weights instead.
#include "block_fp8.h"

#include "block.h"
#include "block_few.h"
#include "block_gemm.h"
#include "block_steps.h"

namespace cconv {
namespace {

void plan(Steps& st, const cconv_fp8_product_args& args) {
  const int64_t M = args.M, N = args.N, K = args.K;
  const Mat a(args.a), b(args.b), sa(args.a_scale), sb(args.b_scale), c(args.c);
  const int dtype = args.dtype, sms = st.sms();
  if (M <= kFewTokens && few_readable(a, M, K, 1) && few_readable(b, N, K, 1)) {
    st.add([=](cudaStream_t s) {
      return block_cuda_error(run_few_fp8(a, b, sa, sb, c, M, N, K, dtype, sms, s), "cconv_few_kernel");
    });
    return;
  }
  Launch l;
  l.epilogue = kScaled;
  l.dtype = dtype;
  l.row_scale = sa;
  l.col_scale = sb;
  l.of[0].M = M;
  l.of[0].N = N;
  l.of[0].K = K;
  l.of[0].a[0] = st.operand(a, M, K);
  l.of[0].b[0] = st.operand(b, N, K);
  choose_cut(&l, sms, false);
  const Mat to[3] = {c, Mat(), Mat()};
  st.launch(l, to);
}

}  // namespace

int64_t fp8_workspace(const cconv_fp8_product_args& a, int sms) {
  Steps st(nullptr, sms, 1, a.dtype);
  plan(st, a);
  return st.bytes();
}

int run_fp8(const cconv_fp8_product_args& a, int sms, cudaStream_t s) {
  Steps st(a.workspace, sms, 1, a.dtype);
  plan(st, a);
  return st.run(s);
}

}  // namespace cconv
