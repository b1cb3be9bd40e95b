// Copies of small operands with zeros behind their rows: a launch for all of a call (with a memset and a copy each, odd
// channels cost a mixture of 30 us 5 to 8 us more).
#include "block_pad.h"

#include <algorithm>

#include "block_device.cuh"
#include "block_few.h"
#include "block_launch.h"

namespace cconv {
namespace {

struct PadParams {
  PaddedCopy of[kMostPadded];
};

// Rows by blockIdx.x, operands by blockIdx.y.
__global__ void __launch_bounds__(256) cconv_pad_kernel(const PadParams p) {
  start_in_order();
  const PaddedCopy& c = p.of[blockIdx.y];
  for (int64_t r = blockIdx.x; r < c.rows; r += gridDim.x) {
    const uint16_t* from = static_cast<const uint16_t*>(c.from.p) + r * c.from.rs;
    uint16_t* to = static_cast<uint16_t*>(const_cast<void*>(c.to.p)) + r * c.to.rs;
    for (int64_t i = threadIdx.x; i < c.to.rs; i += 256) to[i] = i < c.cols ? from[i * c.from.cs] : uint16_t(0);
  }
}

}  // namespace

cudaError_t run_padded_copies(const PaddedCopy* copies, int n, cudaStream_t s) {
  PadParams p{};
  int64_t rows = 1;
  for (int i = 0; i < n; ++i) {
    p.of[i] = copies[i];
    rows = std::max(rows, copies[i].rows);
  }
  return launch(cconv_pad_kernel, dim3(unsigned(std::min<int64_t>(rows, 65536)), unsigned(n)), 256, 0, 1, s, p);
}

Mat Padded::readable(Steps& st, const cconv_matrix& m, int64_t rows, int64_t cols, int64_t* k) {
  *k = cols;
  if (few_readable(Mat(m), rows, cols, 2)) return Mat(m);
  PaddedCopy& c = copies_[n_++];
  c.from = Mat(m);
  c.to = st.scratch(rows, cols, 2);
  c.rows = rows;
  c.cols = cols;
  *k = c.to.rs;
  return c.to;
}

void Padded::add(Steps& st) const {
  if (n_ == 0) return;
  const Padded all = *this;
  st.add([all](cudaStream_t s) { return block_cuda_error(run_padded_copies(all.copies_, all.n_, s), "cconv_pad_kernel"); });
}

}  // namespace cconv
