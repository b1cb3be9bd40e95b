// Products of the feed-forward block: what a launch computes, and the launchers.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "block.h"
#include "block_tma.h"

namespace cconv {

// What becomes of a tile's sums.
enum : int {
  kStore = 0,          // out[0]
  kGated = 1,          // columns are pairs g, u: out[0] = act(g) * u, and out[1] = g, out[2] = u if saved
  kGatedBackward = 2,  // sums are dh; in[0] = g, in[1] = u: out[0] = dg, out[1] = du, out[2] = h
  kPartial = 3,        // fp32 sums of a share of k go to the table of partial sums
  kScaled = 4,         // 8-bit operands, scaled sums: out[0]
  kScaledPartial = 5,  // 8-bit operands, scaled sums of a share of k go to the table
};

// C[m][n] = sum_k A[m][k] B[n][k] by pairs of CTAs.  With two operands a[0], a[1] (and b[0], b[1]):
//   segments  C = A0 B0^T + A1 B1^T                      (equal shapes)
//   stacked   C0 = A0 B^T, C1 = A1 B^T                    (equal shapes; rows of tiles of both)
//   paired    G = A B0^T, U = A B1^T                      (kGated)
struct Product {
  Operand a[2], b[2];
  bool segments = false, stacked = false, paired = false;
  int epilogue = kStore;
  int64_t M = 0, N = 0, K = 0;   // of one product; paired: N = rows of b[0]
  int dtype = 0, act = 0;
  bool save = false;
  Mat out[3], in[2];             // row-major, in place for the copy engine
  // 8-bit operands: scale (i, kb) of rows and columns; i is a row (column) of one token, or 128 of weights:
  // kScaled: rows are tokens; kScaledPartial: columns are
  Mat row_scale, col_scale;
  // kPartial: share s of k of element (m, n) goes to partial[s * slice + n * pitch + m'], where m'
  // counts rows of tiles of both products when stacked
  float* partial = nullptr;
  int64_t pitch = 0, slice = 0;
  int splits = 1;
  int block_n = 256;             // columns of a tile: 256, 128, or (kPartial, b k-contiguous) 64, 32
};

cudaError_t run_product(const Product& p, int sms, bool chained, bool more, cudaStream_t s, int* rc);

// Rows of the partial table that a product of M rows (of each of `stack` products) takes.
int64_t partial_rows(int64_t M, int stack);

// Finishing passes: element (t, f) is the sum over s of partial[s * slice + t * pitch + f].
struct Partial {
  const float* p;
  int64_t pitch, slice;
  int splits;
  int64_t second;  // where the second of two stacked products begins
};
cudaError_t finish_store(const Partial& p, const Mat& out, int64_t M, int64_t N, int dtype, bool more, cudaStream_t s);
cudaError_t finish_gated(const Partial& p, const Mat& gate_pre, const Mat& up_pre, const Mat& h, int64_t M, int64_t N,
                         int act, int dtype, bool more, cudaStream_t s);
cudaError_t finish_gated_backward(const Partial& p, const Mat& gate_pre, const Mat& up_pre, const Mat& dg,
                                  const Mat& du, const Mat& h, int64_t M, int64_t N, int act, int dtype, bool more,
                                  cudaStream_t s);

// Copies rows x cols elements of es bytes between any two layouts.
cudaError_t run_copy(const Mat& from, const Mat& to, int64_t rows, int64_t cols, int es, bool chained, bool more,
                     cudaStream_t s);

// The status word that the product kernels of the current device share (device address).
int block_status_word(int** word);
// Limit of every wait on the device: CCONV_WAIT_LIMIT_MS, by default a second.
uint64_t block_wait_limit_ns();

}  // namespace cconv
