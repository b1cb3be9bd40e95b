// The gated feed-forward block as a sequence of launches.
//
//   forward   [g u] = x [Wg Wu]^T, h = act(g) u       one product with two B operands, h from its epilogue
//             y = h Wd^T
//   backward  dh = dy Wd; dg, du, h from its epilogue, which reads g and u
//             dx = dg Wg + du Wu                       one product, k running over both halves
//             dWg = dg^T x, dWu = du^T x, dWd = dy^T h
//             the last four in one launch where their tiles together fill the SMs better than apart
//
// Up to 16 tokens go through the kernels that stream the weights instead (forward).
#include "block_ffn.h"

#include <algorithm>

#include "block.h"
#include "block_few.h"
#include "block_gemm.h"
#include "block_steps.h"

namespace cconv {
namespace {

Product product(int64_t M, int64_t N, int64_t K) {
  Product p;
  p.M = M;
  p.N = N;
  p.K = K;
  return p;
}

Launch launch_of(const cconv_ffn_args& a, const Product& p, int epilogue) {
  Launch l;
  l.of[0] = p;
  l.epilogue = epilogue;
  l.dtype = a.dtype;
  l.act = a.act;
  return l;
}

Operand in_place(const Mat& m, int64_t rows, int64_t k) {  // scratch: always
  Operand o;
  operand_in_place(m, rows, k, 2, true, &o);
  return o;
}

void forward(Steps& st, const cconv_ffn_args& a) {
  const int64_t T = a.T, D = a.D, F = a.F;
  const int dtype = a.dtype, act = a.act, sms = st.sms();
  const Mat h = st.scratch(T, F, 2), x(a.x), wg(a.w_gate), wu(a.w_up), wd(a.w_down), gate_pre(a.gate_pre), up_pre(a.up_pre),
            out(a.out);
  const bool few = T <= kFewTokens && few_readable(x, T, D, 2) && few_readable(wg, F, D, 2) && few_readable(wu, F, D, 2);
  const bool few_down = T <= kFewTokens && few_readable(wd, D, F, 2);  // (F % 8 == 0: h is readable too)
  // h is rounded to the type (fp16: beyond 65504 it is infinite), since the matrix instructions take nothing longer at
  // their rate: with more than 4 tokens the result is 0.0023 of its norm off in bf16, 0.00029 in fp16, where rounding
  // the result alone leaves 0.0017 and 0.00021; a second product for the rest would double its time.  They work on 8
  // tokens at a time, so up to 4 leave room for what the rounding left, which is multiplied too: for one token
  // the error falls from 1.4 times that of rounding the result alone to 1.0 times, in the same time.  (For 5 to 8
  // it takes a second pass, 27.7 instead of 24.7 us at 2048 x 8192, which is not done.)
  const Mat h_lo = few && few_down && T <= kFewTokensInParts ? st.scratch(T, F, 2) : Mat();
  if (few) {
    st.add([=](cudaStream_t s) {
      return block_cuda_error(run_few_gated(x, wg, wu, gate_pre, up_pre, h, h_lo, T, F, D, act, dtype, sms, s), "cconv_few_kernel");
    });
  } else {
    Product p = product(T, F, D);
    p.paired = true;
    p.a[0] = st.operand(x, T, D);
    st.operands(wg, wu, F, D, &p.b[0], &p.b[1]);
    Launch l = launch_of(a, p, kGated);
    l.save = gate_pre.p != nullptr;
    choose_cut(&l, sms, false);
    const Mat to[3] = {h, l.save ? gate_pre : Mat(), l.save ? up_pre : Mat()};
    st.launch(l, to);
  }
  if (few_down) {
    st.add([=](cudaStream_t s) {
      return block_cuda_error(run_few_product(h, h_lo, wd, out, T, D, F, dtype, sms, few, s), "cconv_few_kernel");
    });
    return;
  }
  Product p = product(T, D, F);
  p.a[0] = in_place(h, T, F);
  p.b[0] = st.operand(wd, D, F);
  Launch l = launch_of(a, p, kStore);
  choose_cut(&l, sms, true);
  const Mat to[3] = {out, Mat(), Mat()};
  st.launch(l, to);
}

void backward(Steps& st, const cconv_ffn_args& a) {
  const int64_t T = a.T, D = a.D, F = a.F;
  const int sms = st.sms();
  // dg, du and h are operands of the tensor cores, rounded to the type as h is above, with the same errors.
  const Mat h = st.scratch(T, F, 2), dg = st.scratch(T, F, 2), du = st.scratch(T, F, 2);
  const Mat dout(a.dout), x(a.x);
  {
    Product p = product(T, F, D);
    p.a[0] = st.operand(dout, T, D, false, &a.dout);
    p.b[0] = st.operand(Mat(a.w_down).t(), F, D);
    p.in[0] = st.readable(a.gate_pre, T, F);
    p.in[1] = st.readable(a.up_pre, T, F);
    Launch l = launch_of(a, p, kGatedBackward);
    choose_cut(&l, sms, false);
    const Mat to[3] = {dg, du, h};
    st.launch(l, to);
  }
  // dx, dw_gate, dw_up, dw_down
  Product ps[4] = {product(T, D, F), product(F, D, T), product(F, D, T), product(D, F, T)};
  const Mat to[4] = {Mat(a.dx), Mat(a.dw_gate), Mat(a.dw_up), Mat(a.dw_down)};
  ps[0].segments = true;
  ps[0].a[0] = in_place(dg, T, F);
  ps[0].a[1] = in_place(du, T, F);
  st.operands(Mat(a.w_gate).t(), Mat(a.w_up).t(), D, F, &ps[0].b[0], &ps[0].b[1]);
  ps[1].a[0] = in_place(dg.t(), F, T);
  ps[2].a[0] = in_place(du.t(), F, T);
  ps[1].b[0] = ps[2].b[0] = st.operand(x.t(), D, T);
  ps[3].a[0] = st.operand(dout.t(), D, T, false, &a.dout);
  ps[3].b[0] = in_place(h.t(), F, T);

  // each by itself, with its own cut
  Launch single[4];
  double apart[4];
  for (int i = 0; i < 4; ++i) {
    single[i] = launch_of(a, ps[i], kStore);
    choose_cut(&single[i], sms, false);
    apart[i] = launch_clocks(single[i], sms);
  }
  // the products first .. 3 together, uncut, at the tile that suits them best
  auto group_of = [&](int first, double* clocks) {
    Launch best;
    for (int n = 256; n >= 128; n /= 2) {
      Launch l = launch_of(a, ps[first], kStore);
      l.count = 4 - first;
      for (int i = first; i < 4; ++i) {
        l.of[i - first] = ps[i];
        l.of[i - first].block_n = n;
      }
      const double c = launch_clocks(l, sms);
      if (n == 256 || c < *clocks) best = l, *clocks = c;
    }
    return best;
  };
  double all_clocks = 0, weights_clocks = 0;
  const Launch all = group_of(0, &all_clocks), weights = group_of(1, &weights_clocks);
  const double each = apart[0] + apart[1] + apart[2] + apart[3];
  const Mat none[3] = {};
  auto alone = [&](int i) {
    const Mat t[3] = {to[i], none[1], none[2]};
    st.launch(single[i], t);
  };
  if (all_clocks <= each && all_clocks <= apart[0] + weights_clocks) {
    st.launch(all, to);
  } else {
    alone(0);
    if (weights_clocks <= each - apart[0]) st.launch(weights, to + 1);
    else for (int i = 1; i < 4; ++i) alone(i);
  }
}

}  // namespace

int64_t ffn_workspace(const cconv_ffn_args& a, bool backward_pass, int sms) {
  Steps st(nullptr, sms, 2, a.dtype);
  backward_pass ? backward(st, a) : forward(st, a);
  return st.bytes();
}

int run_ffn(const cconv_ffn_args& a, bool backward_pass, int sms, cudaStream_t s) {
  Steps st(a.workspace, sms, 2, a.dtype);
  backward_pass ? backward(st, a) : forward(st, a);
  return st.run(s);
}

}  // namespace cconv
