// 8-bit values (e4m3) and the scale of a block, as the quantiser and the norms with 8-bit results form them.
#pragma once
#include "block_device.cuh"

namespace cconv {
namespace {

constexpr float kMax = 448.0f;

// Four values as e4m3, nearest (ties to even), at most +-448 in size.
__device__ __forceinline__ uint32_t e4m3x4(uint64_t ab, uint64_t cd) {
  const float2 x = halves_of(ab), y = halves_of(cd);
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x.y), "f"(x.x));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y.y), "f"(y.x));
  return uint32_t(lo) | uint32_t(hi) << 16;
}

// x / s, correctly rounded, for one s and many x.  A quotient of its own for each element keeps the
// reciprocal unit busier than HBM (8192 x 4096 bf16: 39 us).  Markstein's method instead (IBM J. Res. Dev. 34, 1990):
// with y = 1/s correctly rounded, q + (x - q s) y is correctly rounded once q is within an ulp, which one
// such step from x y makes it; the residuals are exact in a fused multiply-add.  For x of at most 11 bits the
// first of the two steps is correctly rounded already: all 2^23 x 2^10 pairs of mantissas were compared with the
// quotients (8192 x 4096 bf16: one step less is 1.5 us).  The method needs scales whose reciprocal and residuals
// neither overflow nor underflow; others (and NaN) divide.
__device__ __noinline__ uint64_t divide_pair(uint64_t f, float s) {
  const float2 v = halves_of(f);
  return pair_of(__fdiv_rn(v.x, s), __fdiv_rn(v.y, s));
}
struct Divisor {
  float s;
  uint64_t y2, minus_s2;
  bool quick;
  // of a scale and its reciprocal (a scale of 0, of a block of zeros, divides by 1)
  __device__ __forceinline__ Divisor(float scale, float y) {
    s = scale == 0.0f ? 1.0f : scale;
    y2 = pair_of(y, y);
    minus_s2 = pair_of(-s, -s);
    quick = s > 1e-25f && s < 1e25f;
  }
  template <int kSteps, int N>
  __device__ __forceinline__ void divide(uint64_t (&f)[N]) const {
    if (quick) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        uint64_t q = mul2(f[i], y2);
        if (kSteps == 2) q = fma2(fma2(q, minus_s2, f[i]), y2, q);
        f[i] = fma2(fma2(q, minus_s2, f[i]), y2, q);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = divide_pair(f[i], s);
    }
  }
};

// The size of a value as an integer of the same order, in which a NaN is the largest.
__device__ __forceinline__ uint32_t size_of(float v) { return __float_as_uint(v) & 0x7fffffffu; }

}  // namespace
}  // namespace cconv
