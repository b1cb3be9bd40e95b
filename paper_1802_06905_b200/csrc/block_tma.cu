// Tensor maps and operand layouts of the feed-forward sub-block's products (host side).
#include "block_tma.h"

#include <string>

#include "host_setup.h"

namespace cconv {

bool operand_in_place(const Mat& m, int64_t rows, int64_t k, int es, bool allow_row_major, Operand* o) {
  o->p = m.p;
  o->rows = rows;
  o->k = k;
  if (reinterpret_cast<uintptr_t>(m.p) & 15u) return false;
  const int64_t unit = 16 / es;
  auto fits = [&](int64_t step, int64_t pitch, int64_t inner, int64_t outer) {
    if (step != 1 && inner != 1) return false;
    o->pitch = outer == 1 ? round_up64(inner, unit) : pitch;  // the pitch of a single row is not used
    return o->pitch % unit == 0 && o->pitch >= inner && o->pitch * es < (int64_t(1) << 40);
  };
  if (fits(m.cs, m.rs, k, rows)) {
    o->kmajor = true;
    return true;
  }
  if (allow_row_major && fits(m.rs, m.cs, rows, k)) {
    o->kmajor = false;
    return true;
  }
  return false;
}

int encode_map(CUtensorMap* tm, const void* p, int es, int dtype, int64_t inner, int64_t outer, int64_t pitch,
               int box_inner, int box_outer) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) {
    set_last_cuda_error("cuTensorMapEncodeTiled is not available from this driver");
    return CCONV_ECUDA;
  }
  const cuuint64_t dims[2] = {cuuint64_t(inner), cuuint64_t(outer)};
  const cuuint64_t strides[1] = {cuuint64_t(pitch) * es};
  const cuuint32_t box[2] = {cuuint32_t(box_inner), cuuint32_t(box_outer)};
  const cuuint32_t step[2] = {1, 1};
  const CUtensorMapDataType type = es == 1                     ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                   : es == 4                   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == CCONV_TYPE_BF16  ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                               : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  const CUresult r = enc(tm, type, 2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_last_cuda_error("cuTensorMapEncodeTiled(" + std::to_string(inner) + " x " + std::to_string(outer) + ", pitch " +
                        std::to_string(pitch) + ") failed with CUresult " + std::to_string(int(r)));
    return CCONV_ECUDA;
  }
  return CCONV_OK;
}

}  // namespace cconv
