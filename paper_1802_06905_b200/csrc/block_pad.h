// Copies of small operands to rows that 16 bytes at a time can be read from, with zeros behind their ends.
#pragma once
#include "block_steps.h"

namespace cconv {

struct PaddedCopy {
  Mat from, to;  // of 16-bit elements; `to`: rows at a pitch of its row stride, all of it written
  int64_t rows = 0, cols = 0;
};
constexpr int kMostPadded = 2;  // of one launch
cudaError_t run_padded_copies(const PaddedCopy* copies, int n, cudaStream_t s);

// Collects a call's; readable() gives the operand as it lies or as it will lie once add() has put the copies among the steps.
class Padded {
 public:
  // *k: the elements of a row that may be read, a multiple of 8.
  Mat readable(Steps& st, const cconv_matrix& m, int64_t rows, int64_t cols, int64_t* k);
  void add(Steps& st) const;

 private:
  PaddedCopy copies_[kMostPadded];
  int n_ = 0;
};

}  // namespace cconv
