// A call as a sequence of launches: operands that the kernels can read in place or copies of them, products
// with their cuts, results that the copy engine can write or a place for them.
#pragma once
#include <functional>
#include <vector>

#include "block.h"
#include "block_gemm.h"

namespace cconv {

class Steps {
 public:
  // With no base the workspace is only measured, and nothing may be run.
  Steps(void* base, int sms, int es, int dtype) : ws_(base), sms_(sms), es_(es), dtype_(dtype) {}

  int64_t bytes() const { return ws_.used(); }
  int sms() const { return sms_; }

  // A step launches something and gives a status code.
  using Step = std::function<int(cudaStream_t s)>;
  void add(Step f) {
    flush();
    steps_.push_back(std::move(f));
  }
  int run(cudaStream_t s) {
    flush();
    for (const Step& f : steps_) {
      const int rc = f(s);
      if (rc != CCONV_OK) return rc;
    }
    return CCONV_OK;
  }

  // rows x cols elements of `es` bytes, 16-byte aligned rows.
  Mat scratch(int64_t rows, int64_t cols, int es) {
    const int64_t pitch = round_up64(cols, 16 / es);
    return Mat(ws_.take(rows * pitch * es), pitch, 1);
  }
  // Copies of rows gather until the next step and go in one launch (none of them reads what another writes).
  void copy(const Mat& from, const Mat& to, int64_t rows, int64_t cols, int es) {
    if (rows == 0 || cols == 0) return;
    Copy c;
    c.from = from;
    c.to = to;
    c.rows = rows;
    c.cols = cols;
    c.es = es;
    if (copies_rows(from, to)) {
      if (pending_.size() == size_t(kMostCopies)) flush();
      pending_.push_back(c);
    } else {
      steps_.push_back([=](cudaStream_t s) { return block_cuda_error(run_copy(c, s), "cconv_copy_kernel"); });
    }
  }

  // An operand of a product (rows x k) as it lies, or a copy of it: in its own order, where the product takes that
  // and the copies need not transpose, else with k contiguous.  `of` names the argument that `m` is, or is the
  // transpose of (null: used once): one copy of it in one order serves both.  (By the argument and not by the
  // address, so that the workspace does not depend on which arguments share one.)
  Operand copied(const Mat& m, int64_t rows, int64_t k, bool want_kmajor, const void* of) {
    const bool kmajor = want_kmajor || es_ != 2 || m.rs != 1 || m.cs == 1;
    const Mat from = kmajor ? m : m.t();
    const int64_t outer = kmajor ? rows : k, inner = kmajor ? k : rows;
    Mat to;
    for (const Made& c : made_)
      if (of && c.of == of && c.rows == outer && c.cols == inner && c.rs == from.rs && c.cs == from.cs) to = c.to;
    if (!to.rs) {
      to = scratch(outer, inner, es_);
      copy(from, to, outer, inner, es_);
      made_.push_back({of, outer, inner, from.rs, from.cs, to});
    }
    Operand o;
    o.p = to.p;
    o.pitch = to.rs;
    o.kmajor = kmajor;
    o.rows = rows;
    o.k = k;
    return o;
  }
  Operand operand(const Mat& m, int64_t rows, int64_t k, bool want_kmajor = false, const void* of = nullptr) {
    Operand o;
    return operand_in_place(m, rows, k, es_, !want_kmajor && es_ == 2, &o) ? o : copied(m, rows, k, want_kmajor, of);
  }
  // Two operands of one product, in the same order.
  void operands(const Mat& a, const Mat& b, int64_t rows, int64_t k, Operand* oa, Operand* ob) {
    *oa = operand(a, rows, k);
    *ob = operand(b, rows, k, oa->kmajor);
    if (oa->kmajor != ob->kmajor) *oa = copied(a, rows, k, true, nullptr);
  }
  // A matrix that is read row by row.
  Mat readable(const cconv_matrix& m, int64_t rows, int64_t cols) {
    Operand o;
    if (operand_in_place(Mat(m), rows, cols, es_, false, &o)) return Mat(o.p, o.pitch, 1);
    const Mat to = scratch(rows, cols, es_);
    copy(Mat(m), to, rows, cols, es_);
    return to;
  }

  // Adds a launch.  `to[i]` is where out[i] of the i-th product (or of the only one) belongs (Mat(): nowhere; an
  // address may be null while the workspace is measured); what the copy engine cannot write there in place goes
  // to the workspace first.
  void launch(Launch l, const Mat* to) {
    struct Move { Mat from, to; int64_t M, N; };
    std::vector<Move> moves;
    const int es = type_bytes(dtype_);
    for (int i = 0; i < (l.count > 1 ? l.count : 3); ++i) {
      if (!to[i].p && !to[i].rs && !to[i].cs) continue;
      Product& p = l.of[l.count > 1 ? i : 0];
      Mat& out = p.out[l.count > 1 ? 0 : i];
      out = to[i];
      Operand o;
      if (l.cut()) continue;  // written straight to any layout
      // (the copy engine stops a store at the row's last 16 bytes, not at its last element: a row that ends within
      // them would take zeros behind its end)
      if (p.N * es % 16 == 0 && operand_in_place(to[i], p.M, p.N, es, false, &o)) {
        out = Mat(o.p, o.pitch, 1);
      } else {
        out = scratch(p.M, p.N, es);
        moves.push_back({out, to[i], p.M, p.N});
      }
    }
    const int sms = sms_;
    add([=](cudaStream_t s) { return run_products(l, sms, s); });
    for (const Move& m : moves) copy(m.from, m.to, m.M, m.N, es);
  }

 private:
  void flush() {
    if (pending_.empty()) return;
    std::vector<Copy> all;
    all.swap(pending_);
    steps_.push_back([all](cudaStream_t s) {
      return block_cuda_error(run_row_copies(all.data(), int(all.size()), s), "cconv_copy_rows_kernel");
    });
  }

  Carver ws_;
  const int sms_, es_, dtype_;
  std::vector<Step> steps_;
  std::vector<Copy> pending_;  // to be launched
  struct Made {                // a copy of an operand
    const void* of;
    int64_t rows, cols, rs, cs;
    Mat to;
  };
  std::vector<Made> made_;
};

}  // namespace cconv
