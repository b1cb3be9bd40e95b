// The residual-norm kernels' parameters and launchers.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace cconv {

struct NormParams {
  int64_t T;
  int D;
  int nb;  // blocks that have rows of their own (backward: at most T)
  float scale, eps;
  int64_t rows_per_gate;  // 0: one gate row for all tokens
  const void *resid, *block, *gate, *w_post, *w_pre, *dresid_out, *dnorm_out;
  void *resid_out, *norm_out, *dresid, *dblock, *dgate, *dw_post, *dw_pre;
  int64_t resid_rs, block_rs, gate_rs, resid_out_rs, norm_out_rs, dresid_out_rs, dnorm_out_rs, dresid_rs,
      dblock_rs, dgate_rs;
  int sums_by_group;
  int ring_rows;    // rows of the shared-memory ring
  int parts;        // blocks of a cluster that share a row
  uint32_t ring_slot;  // bytes of a row of one array there, where rows begin anywhere
  int* status;      // where a bounded wait that ran out is noted
  uint64_t limit_ns;
  float* part;  // backward: [nb][4][D], and [nb][D] more for rows that registers cannot hold
};

int norm_backward_blocks(int64_t T, int64_t D, int es, int sms);
cudaError_t run_norm_forward(const NormParams& p, int dtype, int sms, cudaStream_t s);
cudaError_t run_norm_backward(const NormParams& p, int dtype, cudaStream_t s);

}  // namespace cconv
