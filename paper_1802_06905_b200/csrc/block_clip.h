// The norm of a list of gradients and their clipping: launches.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "block.h"

namespace cconv {

// Tensors are lists of rows (checked by the caller); those without elements are passed over.
int64_t clip_workspace(const cconv_clip_args& a, int sms);
// Partial sums of squares to the workspace; how many, to *sums.
int run_square_sums(const cconv_clip_args& a, int sms, int* sums, cudaStream_t s);
// The norm from them to a.norm.
int run_norm_of_sums(const cconv_clip_args& a, int sums, cudaStream_t s);
// The results; the norm from the partial sums (which writes it to a.norm) or, if it is given, from a.norm.
int run_clip(const cconv_clip_args& a, int sms, int sums, cudaStream_t s);

}  // namespace cconv
