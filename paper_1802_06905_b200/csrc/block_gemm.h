// Products on pairs of CTAs: what a launch computes, how it is cut, and the launcher.
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
  kScaled = 3,         // 8-bit operands, sums of each block of 128 scaled: out[0]
};

constexpr int kMostProducts = 4;  // of one launch

// C[m][n] = sum_k A[m][k] B[n][k].  With two operands of a kind:
//   segments  C = A0 B0^T + A1 B1^T         (equal shapes and orders)
//   paired    G = A B0^T, U = A B1^T        (kGated)
struct Product {
  Operand a[2], b[2];
  bool segments = false, paired = false;
  int64_t M = 0, N = 0, K = 0;  // paired: N = rows of b[0]
  Mat out[3], in[2];            // `in` row-major; unless cut, all row-major and in place for the copy engine
  int block_n = 256;            // columns of a tile: 256, 128 or (kStore, B k-contiguous) 64
};

struct Launch {
  Product of[kMostProducts];
  int count = 1;                // more than one: kStore, uncut
  int epilogue = kStore;
  int splits = 1;               // pairs that share a tile, each a part of k: 1, 2 or 4
  int dtype = 0, act = 0;
  bool save = false;
  Mat row_scale, col_scale;     // kScaled: scale (row, kb) of A, (row / 128, kb) of B
  bool cut() const { return splits > 1; }  // results then go straight to any layout
};

int run_products(const Launch& l, int sms, cudaStream_t s);

// An estimate of the launch's time in clocks, and the cut that makes it least (`few_columns`: 64 is allowed).
double launch_clocks(const Launch& l, int sms);
void choose_cut(Launch* l, int sms, bool few_columns);

// A copy of rows x cols elements of es bytes from one layout to another.
struct Copy {
  Mat from, to;
  int64_t rows = 0, cols = 0;
  int es = 2;
};
constexpr int kMostCopies = 6;  // of one launch
bool copies_rows(const Mat& from, const Mat& to);  // rows contiguous on both sides
cudaError_t run_row_copies(const Copy* copies, int n, cudaStream_t s);  // at most kMostCopies such
cudaError_t run_copy(const Copy& c, cudaStream_t s);                     // any layouts

// The status word that the product kernels of the current device share (device address).
int block_status_word(int** word);
// Limit of every wait on the device: CCONV_WAIT_LIMIT_MS, by default a second.
uint64_t block_wait_limit_ns();

}  // namespace cconv
