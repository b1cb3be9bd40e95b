// Tensor maps and operand layouts of the feed-forward sub-block's products (host side).
#pragma once
#include <cuda.h>

#include <cstdint>

#include "block.h"

namespace cconv {

// An operand of a product as the copy engine reads it: rows of the M or N dimension by k.
// kmajor: element (row, k) at p + row*pitch + k; else ("row-major") at p + k*pitch + row.
struct Operand {
  const void* p = nullptr;
  int64_t pitch = 0;  // elements
  bool kmajor = true;
  int64_t rows = 0, k = 0;
};

// Whether the copy engine can read `m` (rows x k elements of `es` bytes) in place, k contiguous or rows
// contiguous: unit stride, a 16-byte aligned address, a pitch that is a multiple of 16 bytes and at
// least a row long.  Fills *o.
bool operand_in_place(const Mat& m, int64_t rows, int64_t k, int es, bool allow_row_major, Operand* o);

// 2-D tensor map: `inner` contiguous elements by `outer` rows at `pitch` elements; a box of box_inner x
// box_outer with 128-byte swizzle (box_inner * es = 128).  es: 1 (e4m3), 2 (bf16 or fp16 by dtype).  Loads read zeros
// past `inner`; stores write the whole 16 bytes that `inner` ends in.
int encode_map(CUtensorMap* tm, const void* p, int es, int dtype, int64_t inner, int64_t outer, int64_t pitch,
               int box_inner, int box_outer);

}  // namespace cconv
