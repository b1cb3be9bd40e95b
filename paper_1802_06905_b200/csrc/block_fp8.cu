// The 8-bit product with a scale for each block of 128, as a sequence of launches.
//
// C[m][n] = sum_kb sa[m][kb] sb[n/128][kb] (A B^T)_kb: the tensor cores form the sums of one block of 128
// (one stage: 128 bytes of k a row), which the epilogue warps scale and add up in fp32 registers while the
// next block's are formed.  Few tokens, or few tiles: cut along k, as in the feed-forward block.
#include "block_fp8.h"

#include <algorithm>

#include "block.h"
#include "block_few.h"
#include "block_gemm.h"

namespace cconv {
namespace {

class Runner {
 public:
  Runner(const cconv_fp8_product_args& a, int sms, void* base, bool dry, int launches, cudaStream_t s)
      : a_(a), sms_(sms), ws_(base), dry_(dry), launches_(launches), s_(s) {}
  int rc = CCONV_OK;
  int made = 0;
  int64_t bytes() const { return ws_.used(); }

  void run() {
    const int pairs = sms_ / 2;
    const int64_t M = a_.M, N = a_.N, K = a_.K, kb = cdiv64(K, 128);
    const int64_t tiles = cdiv64(M, 256) * cdiv64(N, 128);
    if (M <= kFewTokens && few_readable(Mat(a_.a), M, K, 1) && few_readable(Mat(a_.b), N, K, 1)) {
      launch([&](bool) {
        return run_few_fp8(Mat(a_.a), Mat(a_.b), Mat(a_.a_scale), Mat(a_.b_scale), Mat(a_.c), M, N, K, a_.dtype, sms_, s_);
      });
      return;
    }
    Product p;
    p.K = K;
    p.dtype = a_.dtype;
    const Operand ta = operand(Mat(a_.a), M, K), tb = operand(Mat(a_.b), N, K);
    if (M <= 128 || (2 * tiles <= pairs && kb >= 8)) {
      p.epilogue = kScaledPartial;
      p.M = N;
      p.N = M;
      p.a[0] = tb;
      p.b[0] = ta;
      p.row_scale = Mat(a_.b_scale);
      p.col_scale = Mat(a_.a_scale);
      p.block_n = M <= 32 ? 32 : M <= 64 ? 64 : M <= 128 ? 128 : 256;
      const int64_t t = cdiv64(N, 256) * cdiv64(M, p.block_n);
      const int64_t want = std::max<int64_t>(1, std::min<int64_t>(pairs / t, kb / 4));
      p.splits = int(cdiv64(kb, cdiv64(kb, want)));
      p.pitch = partial_rows(N, 1);
      p.slice = M * p.pitch;
      p.partial = static_cast<float*>(ws_.take(p.slice * p.splits * 4));
      launch([&](bool more) { return product(p, more); });
      const Partial part{p.partial, p.pitch, p.slice, p.splits, 0};
      launch([&](bool more) { return finish_store(part, Mat(a_.c), M, N, a_.dtype, more, s_); });
      return;
    }
    p.epilogue = kScaled;
    p.M = M;
    p.N = N;
    p.a[0] = ta;
    p.b[0] = tb;
    p.row_scale = Mat(a_.a_scale);
    p.col_scale = Mat(a_.b_scale);
    const int64_t m = cdiv64(M, 256);
    p.block_n = double(cdiv64(m * cdiv64(N, 128), pairs)) * 1.15 < double(cdiv64(m * cdiv64(N, 256), pairs)) * 2 ? 128 : 256;
    Operand o;
    const int es = type_bytes(a_.dtype);
    const bool direct = operand_in_place(Mat(a_.c), M, N, es, false, &o);
    p.out[0] = Mat(o.p, o.pitch, 1);
    if (!direct) {
      const int64_t pitch = round_up64(N, 16 / es);
      p.out[0] = Mat(ws_.take(M * pitch * es), pitch, 1);
    }
    launch([&](bool more) { return product(p, more); });
    if (!direct) launch([&](bool more) { return run_copy(p.out[0], Mat(a_.c), M, N, es, true, more, s_); });
  }

 private:
  Operand operand(const Mat& m, int64_t rows, int64_t k) {
    Operand o;
    if (operand_in_place(m, rows, k, 1, false, &o)) return o;
    o.pitch = round_up64(k, 16);
    o.p = ws_.take(rows * o.pitch);
    o.kmajor = true;
    launch([&](bool more) { return run_copy(m, Mat(o.p, o.pitch, 1), rows, k, 1, made > 0, more, s_); });
    return o;
  }
  cudaError_t product(const Product& p, bool more) {
    int code = CCONV_OK;
    const cudaError_t e = run_product(p, sms_, made > 0, more, s_, &code);
    if (code != CCONV_OK) rc = code;
    return e;
  }
  template <typename F>
  void launch(F f) {
    if (!dry_ && rc == CCONV_OK) {
      const int code = block_cuda_error(f(made + 1 < launches_), "cconv_fp8_product");
      if (rc == CCONV_OK) rc = code;
    }
    ++made;
  }

  const cconv_fp8_product_args& a_;
  const int sms_;
  Carver ws_;
  const bool dry_;
  const int launches_;
  cudaStream_t s_;
};

}  // namespace

int64_t fp8_workspace(const cconv_fp8_product_args& a, int sms) {
  Runner r(a, sms, nullptr, true, 0, nullptr);
  r.run();
  return r.bytes();
}

int run_fp8(const cconv_fp8_product_args& a, int sms, cudaStream_t s) {
  Runner count(a, sms, a.workspace, true, 0, s);
  count.run();
  Runner r(a, sms, a.workspace, false, count.made, s);
  r.run();
  return r.rc;
}

}  // namespace cconv
