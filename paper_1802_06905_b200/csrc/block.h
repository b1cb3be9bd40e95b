// Host-side pieces shared by the entry points of the feed-forward sub-block (include/cconv_block.h).
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/cconv_block.h"

namespace cconv {

// A matrix operand as the kernels see it: address of element (0,0), strides in elements.
struct Mat {
  const void* p = nullptr;
  int64_t rs = 0, cs = 0;
  Mat() = default;
  Mat(const void* p_, int64_t rs_, int64_t cs_) : p(p_), rs(rs_), cs(cs_) {}
  explicit Mat(const cconv_matrix& m) : p(m.data), rs(m.row_stride), cs(m.col_stride) {}
  Mat t() const { return Mat(p, cs, rs); }
};

inline int64_t cdiv64(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up64(int64_t a, int64_t b) { return cdiv64(a, b) * b; }
inline int type_bytes(int dtype) { return dtype == CCONV_TYPE_FP32 ? 4 : 2; }

// Carves 256-byte aligned pieces out of a workspace; with no base it only adds up their sizes.
class Carver {
 public:
  explicit Carver(void* base) : base_(static_cast<char*>(base)) {}
  void* take(int64_t bytes) {
    char* p = base_ ? base_ + used_ : nullptr;
    used_ += round_up64(bytes, 256);
    return p;
  }
  int64_t used() const { return used_; }

 private:
  char* base_;
  int64_t used_ = 0;
};

// SMs of the current device (cached per device), or a negative code with the error text set.
int block_sm_count();
int block_cuda_error(cudaError_t e, const char* where);

// Kernels and memsets that this host thread has put into streams for the sub-block, so far.
int64_t& block_launches();

}  // namespace cconv
