// Quantisation to e4m3 in blocks of 128 channels, of one token (activations) or of 128 rows (weights).
//
//   scale = max|x| / 448,  q = e4m3(x / scale), nearest, ties to even
//
// One pass: the values of a block stay in registers between its maximum and its rounding.  Bound by HBM:
// 2 bytes read and 1 written an element (16-bit x).  Both quotients are IEEE divisions, so that
// the result is the definition's bit for bit.
#include <cuda_fp8.h>

#include <algorithm>

#include "block.h"
#include "block_device.cuh"
#include "block_quant.h"

namespace cconv {
namespace {

constexpr float kMax = 448.0f;

// max that keeps a NaN (fmaxf would drop it)
__device__ __forceinline__ float max_nan(float a, float b) { return (a > b || a != a) ? a : b; }

__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return uint32_t(lo) | uint32_t(hi) << 16;
}

// Eight elements from p, of which the first n are in range (kWide: all or, n <= 0, none).
template <typename T, bool kWide>
__device__ __forceinline__ void load8(float (&f)[8], const T* p, int64_t cs, int64_t n) {
  if constexpr (kWide && sizeof(T) == 2) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (n > 0) w = *reinterpret_cast<const uint4*>(p);
    const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y), c = unpack2<T>(w.z), d = unpack2<T>(w.w);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? to_f32(p[i * cs]) : 0.0f;
  }
}

// 16 lanes a 128-channel group, 8 channels a lane; kRows groups (rows) a lane: 1 (a block is one token's
// group) or 8 (a CTA of 256 threads takes 16 x 8 = 128 rows).
template <typename T, int kRows, bool kWide>
__global__ void __launch_bounds__(256) cconv_quantize_kernel(const QuantParams p) {
  __shared__ float smem[8];
  const T* x = static_cast<const T*>(p.x);
  const int sub = threadIdx.x & 15, row_in = threadIdx.x >> 4;
  for (int64_t b = blockIdx.x; b < p.blocks; b += gridDim.x) {
    const int64_t cb = b % p.col_blocks, rb = b / p.col_blocks;
    const int64_t c = cb * 128 + sub * 8;
    float f[kRows][8];
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int64_t t = (rb * kRows + i) * 16 + row_in;
      load8<T, kWide>(f[i], x + t * p.x_rs + c * p.x_cs, p.x_cs, t < p.T ? p.D - c : 0);
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max_nan(fabsf(f[i][j]), m);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max_nan(__shfl_xor_sync(0xffffffffu, m, o), m);
    if (kRows > 1) {
      m = max_nan(__shfl_xor_sync(0xffffffffu, m, 16), m);
      if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = m;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max_nan(smem[i], m);
      __syncthreads();
    }
    const float scale = __fdiv_rn(m, kMax);
    const float by = scale == 0.0f ? 1.0f : scale;
    if (kRows > 1) {
      if (threadIdx.x == 0) p.scale[rb * p.scale_rs + cb * p.scale_cs] = scale;
    } else if (sub == 0 && rb * 16 + row_in < p.T) {
      p.scale[(rb * 16 + row_in) * p.scale_rs + cb * p.scale_cs] = scale;
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int64_t t = (rb * kRows + i) * 16 + row_in;
      if (t >= p.T) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = __fdiv_rn(f[i][j], by);
      const uint32_t lo = e4m3x4(f[i][0], f[i][1], f[i][2], f[i][3]);
      const uint32_t hi = e4m3x4(f[i][4], f[i][5], f[i][6], f[i][7]);
      uint8_t* q = p.q + t * p.q_rs + c * p.q_cs;
      if (kWide) {
        if (c < p.D) *reinterpret_cast<uint2*>(q) = make_uint2(lo, hi);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < p.D) q[j * p.q_cs] = uint8_t((j < 4 ? lo : hi) >> (8 * (j & 3)));
      }
    }
  }
}

template <typename T>
cudaError_t launch(QuantParams p, int block_rows, int sms, cudaStream_t s) {
  const uintptr_t in = reinterpret_cast<uintptr_t>(p.x) | uintptr_t(p.x_rs * int64_t(sizeof(T)));
  const uintptr_t out = reinterpret_cast<uintptr_t>(p.q) | uintptr_t(p.q_rs);
  const bool wide = sizeof(T) == 2 && p.D % 8 == 0 && p.x_cs == 1 && p.q_cs == 1 && (in & 15) == 0 && (out & 7) == 0;
  p.col_blocks = cdiv64(p.D, 128);
  p.blocks = p.col_blocks * cdiv64(p.T, block_rows == 1 ? 16 : 128);
  const unsigned grid = unsigned(std::min<int64_t>(p.blocks, int64_t(sms) * 64));
  if (block_rows == 1) {
    if (wide) cconv_quantize_kernel<T, 1, true><<<grid, 256, 0, s>>>(p);
    else cconv_quantize_kernel<T, 1, false><<<grid, 256, 0, s>>>(p);
  } else {
    if (wide) cconv_quantize_kernel<T, 8, true><<<grid, 256, 0, s>>>(p);
    else cconv_quantize_kernel<T, 8, false><<<grid, 256, 0, s>>>(p);
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t run_quantize(const QuantParams& p, int dtype, int block_rows, int sms, cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16) return launch<__nv_bfloat16>(p, block_rows, sms, s);
  if (dtype == CCONV_TYPE_FP16) return launch<__half>(p, block_rows, sms, s);
  return launch<float>(p, block_rows, sms, s);
}

}  // namespace cconv
