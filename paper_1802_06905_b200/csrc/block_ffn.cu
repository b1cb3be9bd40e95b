// The gated feed-forward block as a sequence of launches.
//
//   forward   [g u] = x [Wg Wu]^T, h = act(g) u       one product with two B operands, h from its epilogue
//             y = h Wd^T
//   backward  dh = dy Wd; dg, du, h from its epilogue, which reads g and u
//             dx = dg Wg + du Wu                       one product, k running over both halves
//             dWg = dg^T x, dWu = du^T x               one launch, rows of tiles of both
//             dWd = dy^T h
//
// A product whose tiles would leave most pairs of CTAs without work is cut along k instead: the shares'
// sums go to a table in fp32 and a second launch adds them up in order and does what the epilogue
// would have done.  For few tokens that is every product but those of the weights' gradients; the
// tokens are then the columns of a tile, so that the tile's 256 rows are rows of the weights.
#include "block_ffn.h"

#include <algorithm>

#include "block.h"
#include "block_few.h"
#include "block_gemm.h"

namespace cconv {
namespace {

class Runner {
 public:
  Runner(const cconv_ffn_args& a, int sms, void* base, bool dry, int launches, cudaStream_t s)
      : a_(a), sms_(sms), ws_(base), dry_(dry), launches_(launches), s_(s) {}
  int rc = CCONV_OK;
  int made = 0;  // launches so far
  int64_t bytes() const { return ws_.used(); }

  void forward() {
    const int64_t T = a_.T, D = a_.D, F = a_.F;
    const Mat h = scratch(T, F);
    if (T <= kFewTokens && few_readable(Mat(a_.x), T, D, 2) && few_readable(Mat(a_.w_gate), F, D, 2) &&
        few_readable(Mat(a_.w_up), F, D, 2)) {
      finish([&](bool more) {
        return run_few_gated(Mat(a_.x), Mat(a_.w_gate), Mat(a_.w_up), Mat(a_.gate_pre), Mat(a_.up_pre), h, T, F, D, a_.act,
                             a_.dtype, sms_, more, s_);
      });
      down(h);
      return;
    }
    Result gate_pre, up_pre;
    const bool save = a_.gate_pre.data != nullptr;
    const int64_t tiles = cdiv64(T, 256) * cdiv64(F, 128);
    if (few(T) || 2 * tiles <= pairs()) {
      Product p = base(F, T, D);
      p.stacked = true;
      p.a[0] = operand(Mat(a_.w_gate), F, D);
      p.a[1] = operand(Mat(a_.w_up), F, D, p.a[0].kmajor);
      same_order(p.a[0], p.a[1], Mat(a_.w_gate), Mat(a_.w_up));
      p.b[0] = tokens(Mat(a_.x), T, D, &p.block_n);
      const Partial part = partial(p);
      launch(p);
      finish([&](bool more) {
        return finish_gated(part, Mat(a_.gate_pre), Mat(a_.up_pre), h, T, F, a_.act, a_.dtype, more, s_);
      });
    } else {
      Product p = base(T, F, D);
      p.paired = true;
      p.epilogue = kGated;
      p.a[0] = operand(Mat(a_.x), T, D);
      p.b[0] = operand(Mat(a_.w_gate), F, D);
      p.b[1] = operand(Mat(a_.w_up), F, D, p.b[0].kmajor);
      same_order(p.b[0], p.b[1], Mat(a_.w_gate), Mat(a_.w_up));
      p.save = save;
      p.out[0] = h;
      if (save) {
        gate_pre = result(a_.gate_pre, T, F);
        up_pre = result(a_.up_pre, T, F);
        p.out[1] = gate_pre.at;
        p.out[2] = up_pre.at;
      }
      launch(p);
    }
    down(h);
    place(gate_pre, T, F);
    place(up_pre, T, F);
  }

  void backward() {
    const int64_t T = a_.T, D = a_.D, F = a_.F;
    const Mat h = scratch(T, F), dg = scratch(T, F), du = scratch(T, F);
    const Mat dout(a_.dout), x(a_.x), wd(a_.w_down);
    const int64_t tiles = cdiv64(T, 256) * cdiv64(F, 128);
    if (few(T) || 2 * tiles <= pairs()) {
      Product p = base(F, T, D);
      p.a[0] = operand(wd.t(), F, D);
      p.b[0] = tokens(dout, T, D, &p.block_n);
      const Partial part = partial(p);
      launch(p);
      finish([&](bool more) {
        return finish_gated_backward(part, Mat(a_.gate_pre), Mat(a_.up_pre), dg, du, h, T, F, a_.act, a_.dtype, more, s_);
      });
    } else {
      Product p = base(T, F, D);
      p.epilogue = kGatedBackward;
      p.a[0] = operand(dout, T, D);
      p.b[0] = operand(wd.t(), F, D);
      p.in[0] = readable(a_.gate_pre, T, F);
      p.in[1] = readable(a_.up_pre, T, F);
      p.out[0] = dg;
      p.out[1] = du;
      p.out[2] = h;
      p.block_n = columns(T, F);
      launch(p);
    }
    Operand kg = in_place(dg, T, F), ku = in_place(du, T, F);
    Operand wg = operand(Mat(a_.w_gate).t(), D, F), wu = operand(Mat(a_.w_up).t(), D, F, wg.kmajor);
    same_order(wg, wu, Mat(a_.w_gate).t(), Mat(a_.w_up).t());
    store(&kg, &ku, &wg, &wu, Mat(), T, D, F, a_.dx);
    Operand xt = operand(x.t(), D, T);
    Operand gt = in_place(dg.t(), F, T), ut = in_place(du.t(), F, T);
    const int64_t wtiles = cdiv64(F, 256) * cdiv64(D, 128);
    if (4 * wtiles <= pairs()) {
      store(&gt, nullptr, &xt, nullptr, Mat(), F, D, T, a_.dw_gate);
      store(&ut, nullptr, &xt, nullptr, Mat(), F, D, T, a_.dw_up);
    } else {
      Product p = base(F, D, T);
      p.stacked = true;
      p.a[0] = gt;
      p.a[1] = ut;
      p.b[0] = xt;
      const Result g = result(a_.dw_gate, F, D), u = result(a_.dw_up, F, D);
      p.out[0] = g.at;
      p.out[1] = u.at;
      p.block_n = columns(2 * F, D);
      launch(p);
      place(g, F, D);
      place(u, F, D);
    }
    Operand dt = operand(dout.t(), D, T), ht = in_place(h.t(), F, T);
    store(&dt, nullptr, &ht, nullptr, Mat(), D, F, T, a_.dw_down);
  }

 private:
  struct Result {
    Mat at, to;      // where the kernels write; where it belongs, if elsewhere
    bool move = false;
  };

  int pairs() const { return sms_ / 2; }
  static bool few(int64_t T) { return T <= 128; }

  // y = h Wd^T
  void down(const Mat& h) {
    const int64_t T = a_.T, D = a_.D, F = a_.F;
    if (T <= kFewTokens && few_readable(Mat(a_.w_down), D, F, 2)) {  // (F % 8 == 0: h is readable too)
      finish([&](bool more) {
        return run_few_product(h, Mat(a_.w_down), Mat(a_.out), T, D, F, a_.dtype, sms_, made > 0, more, s_);
      });
      return;
    }
    const Operand hk = in_place(h, T, F);
    store(&hk, nullptr, nullptr, nullptr, Mat(a_.w_down), T, D, F, a_.out);
  }

  Product base(int64_t M, int64_t N, int64_t K) const {
    Product p;
    p.M = M;
    p.N = N;
    p.K = K;
    p.dtype = a_.dtype;
    p.act = a_.act;
    return p;
  }

  // A T x F matrix of the type in the workspace.
  Mat scratch(int64_t rows, int64_t cols) {
    const int64_t pitch = round_up64(cols, 8);
    return Mat(ws_.take(rows * pitch * 2), pitch, 1);
  }
  Operand in_place(const Mat& m, int64_t rows, int64_t k) {
    Operand o;
    operand_in_place(m, rows, k, 2, true, &o);  // scratch: always
    return o;
  }
  Operand copied(const Mat& m, int64_t rows, int64_t k) {
    const Mat to = scratch(rows, k);
    finish([&](bool more) { return run_copy(m, to, rows, k, 2, made > 0, more, s_); });
    Operand o;
    o.p = to.p;
    o.pitch = to.rs;
    o.kmajor = true;
    o.rows = rows;
    o.k = k;
    return o;
  }
  // An operand as it lies, or a copy of it with k contiguous.
  Operand operand(const Mat& m, int64_t rows, int64_t k, bool want_kmajor = false) {
    Operand o;
    if (operand_in_place(m, rows, k, 2, !want_kmajor, &o)) return o;
    return copied(m, rows, k);
  }
  // Two operands of one product lie in the same order.
  void same_order(Operand& a, Operand& b, const Mat& ma, const Mat& mb) {
    if (a.kmajor == b.kmajor) return;
    if (!a.kmajor) a = copied(ma, a.rows, a.k);
    else b = copied(mb, b.rows, b.k);
  }
  // Tokens as the columns of a tile: k contiguous where a tile has fewer than 128.
  Operand tokens(const Mat& m, int64_t T, int64_t k, int* block_n) {
    *block_n = T <= 32 ? 32 : T <= 64 ? 64 : T <= 128 ? 128 : 256;
    return operand(m, T, k, *block_n < 128);
  }
  Mat readable(const cconv_matrix& m, int64_t rows, int64_t cols) {
    Operand o;
    if (operand_in_place(Mat(m), rows, cols, 2, false, &o)) return Mat(o.p, o.pitch, 1);
    const Mat to = scratch(rows, cols);
    finish([&](bool more) { return run_copy(Mat(m), to, rows, cols, 2, made > 0, more, s_); });
    return to;
  }
  // Where the copy engine can write a result of the caller's.
  Result result(const cconv_matrix& m, int64_t rows, int64_t cols) {
    Result r;
    Operand o;
    if (operand_in_place(Mat(m), rows, cols, 2, false, &o)) {
      r.at = Mat(o.p, o.pitch, 1);
      return r;
    }
    r.at = scratch(rows, cols);
    r.to = Mat(m);
    r.move = true;
    return r;
  }
  void place(const Result& r, int64_t rows, int64_t cols) {
    if (r.move) finish([&](bool more) { return run_copy(r.at, r.to, rows, cols, 2, true, more, s_); });
  }

  // Columns of a tile: 128 where they leave fewer idle pairs in the last round than 256 cost in reads
  // (a 256 x 128 tile draws 1.5 times the bytes of L2 a product that a 256 x 256 tile does; taken as
  // 1.15 times the time).
  int columns(int64_t M, int64_t N) const {
    const int64_t m = cdiv64(M, 256);
    const double wide = double(cdiv64(m * cdiv64(N, 256), pairs())) * 2.0;
    const double narrow = double(cdiv64(m * cdiv64(N, 128), pairs())) * 1.15;
    return narrow < wide ? 128 : 256;
  }

  // Cuts the product p (rows: features) along k and gives its table of partial sums.
  Partial partial(Product& p) {
    p.epilogue = kPartial;
    const int stack = p.stacked ? 2 : 1;
    const int64_t tiles = cdiv64(p.M, 256) * stack * cdiv64(p.N, p.block_n);
    const int64_t kb = cdiv64(p.K, 64) * (p.segments ? 2 : 1);
    // at least 4 stages of k a share
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(pairs() / tiles, kb / 4));
    p.splits = int(cdiv64(kb, cdiv64(kb, want)));
    p.pitch = partial_rows(p.M, stack);
    p.slice = p.N * p.pitch;
    p.partial = static_cast<float*>(ws_.take(p.slice * p.splits * 4));
    return Partial{p.partial, p.pitch, p.slice, p.splits, p.pitch / stack};
  }

  // out = A B^T (+ A1 B1^T): B given or `mb`.  M x N results with K (each) terms.
  void store(const Operand* a0, const Operand* a1, const Operand* b0, const Operand* b1, const Mat& mb,
             int64_t M, int64_t N, int64_t K, const cconv_matrix& out) {
    const int64_t tiles = cdiv64(M, 256) * cdiv64(N, 128);
    const int64_t kb = cdiv64(K, 64) * (a1 ? 2 : 1);
    if (few(M) || (2 * tiles <= pairs() && kb >= 8)) {
      // rows of tiles are the result's columns, columns of tiles its rows
      Product p = base(N, M, K);
      p.segments = a1 != nullptr;
      p.a[0] = b0 ? *b0 : operand(mb, N, K);
      if (b1) p.a[1] = *b1;
      p.b[0] = *a0;
      if (a1) p.b[1] = *a1;
      p.block_n = M <= 32 ? 32 : M <= 64 ? 64 : M <= 128 ? 128 : 256;
      if (!a0->kmajor && p.block_n < 128) p.block_n = 128;
      const Partial part = partial(p);
      launch(p);
      finish([&](bool more) { return finish_store(part, Mat(out), M, N, a_.dtype, more, s_); });
      return;
    }
    Product p = base(M, N, K);
    p.segments = a1 != nullptr;
    p.a[0] = *a0;
    if (a1) p.a[1] = *a1;
    p.b[0] = b0 ? *b0 : operand(mb, N, K);
    if (b1) p.b[1] = *b1;
    const Result r = result(out, M, N);
    p.out[0] = r.at;
    p.block_n = columns(M, N);
    launch(p);
    place(r, M, N);
  }

  void launch(const Product& p) {
    if (!dry_ && rc == CCONV_OK) {
      int code = CCONV_OK;
      const cudaError_t e = run_product(p, sms_, made > 0, made + 1 < launches_, s_, &code);
      rc = code != CCONV_OK ? code : block_cuda_error(e, "cconv_pair_product_kernel");
    }
    ++made;
  }
  template <typename F>
  void finish(F f) {
    if (!dry_ && rc == CCONV_OK) rc = block_cuda_error(f(made + 1 < launches_), "feed-forward block");
    ++made;
  }

  const cconv_ffn_args& a_;
  const int sms_;
  Carver ws_;
  const bool dry_;
  const int launches_;
  cudaStream_t s_;
};

}  // namespace

int64_t ffn_workspace(const cconv_ffn_args& a, bool backward, int sms) {
  Runner r(a, sms, nullptr, true, 0, nullptr);
  backward ? r.backward() : r.forward();
  return r.bytes();
}

int run_ffn(const cconv_ffn_args& a, bool backward, int sms, cudaStream_t s) {
  Runner count(a, sms, a.workspace, true, 0, s);
  backward ? count.backward() : count.forward();
  Runner r(a, sms, a.workspace, false, count.made, s);
  backward ? r.backward() : r.forward();
  return r.rc;
}

}  // namespace cconv
