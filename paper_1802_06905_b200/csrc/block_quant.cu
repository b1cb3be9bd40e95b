// Quantisation to e4m3 in blocks of 128 channels, of one token (activations) or of 128 rows (weights).
//
//   scale = max|x| / 448,  q = e4m3(x / scale), nearest, ties to even
//
// One pass: the values of a block stay in registers between its maximum and its rounding.  3 bytes an element
// (16-bit x) pass through HBM, and about 12 instructions of a lane take as long to issue: tokens 8192 x 4096
// bf16 20.6 us, 4.9 TB/s (the bytes alone: 15.4 us); weights 2600 x 2000 5.5 us.  Both quotients are correctly rounded, so
// that the result is the definition's bit for bit.
#include <algorithm>

#include "block.h"
#include "block_device.cuh"
#include "block_e4m3.cuh"
#include "block_launch.h"
#include "block_quant.h"

namespace cconv {
namespace {

template <typename T>
struct Two;
template <>
struct Two<__nv_bfloat16> {
  using type = __nv_bfloat162;
};
template <>
struct Two<__half> {
  using type = __half2;
};

// Eight elements of a row: packed (16-bit types, 16 bytes at once) or one by one, `step` apart in memory.
template <typename T, bool kWide>
struct Eight {
  float f[8];
  __device__ __forceinline__ void load(const T* p, int64_t step, int64_t n) {  // the first n are in range
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? to_f32(p[i * step]) : 0.0f;
  }
  __device__ __forceinline__ void get(uint64_t (&o)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pair_of(f[2 * i], f[2 * i + 1]);
  }
  __device__ __forceinline__ uint32_t largest() const {  // as size_of
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, size_of(f[i]));
    return m;
  }
};
template <typename T>
struct Eight<T, true> {
  uint4 w;
  __device__ __forceinline__ void load(const T* p, int64_t, int64_t n) {  // all are in range or, n <= 0, none
    w = make_uint4(0, 0, 0, 0);
    if (n > 0) w = *reinterpret_cast<const uint4*>(p);
  }
  __device__ __forceinline__ void get(uint64_t (&f)[4]) const {
    const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y), c = unpack2<T>(w.z), d = unpack2<T>(w.w);
    f[0] = pair_of(a.x, a.y);
    f[1] = pair_of(b.x, b.y);
    f[2] = pair_of(c.x, c.y);
    f[3] = pair_of(d.x, d.y);
  }
  __device__ __forceinline__ uint32_t largest() const {
    using T2 = typename Two<T>::type;
    auto size2 = [](uint32_t u) { return __habs2(*reinterpret_cast<const T2*>(&u)); };
    const T2 m = __hmax2_nan(__hmax2_nan(size2(w.x), size2(w.y)), __hmax2_nan(size2(w.z), size2(w.w)));
    const float2 v = unpack2<T>(*reinterpret_cast<const uint32_t*>(&m));
    return max(size_of(v.x), size_of(v.y));
  }
};

// kLanes lanes a row of 128 channels, U rows a lane: pieces of 8 channels, 8 kLanes apart, or, where accesses are of
// one element, every 16th channel, so that the lanes' are neighbours (8192 x 4095 bf16: 44 us; 8 channels a lane:
// 95 us).  kBlock = 1:
// each row has a scale, 256 threads.  kBlock = 128: 512 threads take 128 rows and one scale.
// What a row costs besides its elements (the reduction, the scale, its addresses) keeps the issue slots
// busier than the elements do; 8 lanes a row share it among fewer threads than 16 (tokens 8192 x 4096
// bf16: 1.2 times as long with 16).  Blocks that stay and load their next rows while they work on these
// were no faster (22.6 us with 3 an SM, 24.8 with 4, 23.7 with 4 rows a lane and 2).
template <typename T, int kBlock, int kLanes, int U, bool kWide, bool kUnit>
__global__ void __launch_bounds__(kBlock == 1 ? 256 : 512, U == 2 ? 4 : 1) cconv_quantize_kernel(const QuantParams p) {
  constexpr int kAcross = (kBlock == 1 ? 256 : 512) / kLanes, kPieces = 16 / kLanes;
  static_assert(kBlock == 1 || U * kAcross == 128, "");
  __shared__ uint32_t smem[16];
  start_in_order();
  const T* x = static_cast<const T*>(p.x);
  const int sub = threadIdx.x % kLanes, row_in = threadIdx.x / kLanes;
  constexpr int kStep = kWide ? 1 : kLanes;  // from one of a lane's channels to its next
  const int64_t x_cs = kUnit ? 1 : p.x_cs, q_cs = kUnit ? 1 : p.q_cs;
  static_assert(kWide || kPieces == 1, "");
  const int64_t cb = blockIdx.x, c = cb * 128 + sub * (kWide ? 8 : 1);
  const int cols = (int(min(p.D - c, int64_t(128))) + kStep - 1) / kStep;  // of a lane, from c on; may be negative
  for (int64_t rb = blockIdx.y; rb < p.row_blocks; rb += gridDim.y) {
    const int64_t t0 = rb * U * kAcross + row_in;
    const int rows = int(min(int64_t(U * kAcross), p.T - t0));  // from t0 on; may be negative
    const T* from = x + t0 * p.x_rs + c * x_cs;
    uint8_t* q = p.q + t0 * p.q_rs + c * q_cs;
    float* scales = p.scale + (kBlock == 1 ? t0 : rb) * p.scale_rs + cb * p.scale_cs;
    Eight<T, kWide> v[U][kPieces];
    uint32_t m[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < kPieces; ++j)
        v[i][j].load(from + i * (kAcross * p.x_rs) + j * (8 * kLanes * x_cs), kStep * x_cs, i * kAcross < rows ? cols - j * 8 * kLanes : 0);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      m[i] = v[i][0].largest();
      if (kPieces == 2) m[i] = max(m[i], v[i][kPieces - 1].largest());
    }
    if constexpr (kBlock == 1) {
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < U; ++i) m[i] = max(m[i], __shfl_xor_sync(0xffffffffu, m[i], o));
    } else {
#pragma unroll
      for (int i = 1; i < U; ++i) m[0] = max(m[0], m[i]);
      m[0] = __reduce_max_sync(0xffffffffu, m[0]);
      if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = m[0];
      __syncthreads();
      m[0] = __reduce_max_sync(0xffffffffu, smem[threadIdx.x & 15]);
      __syncthreads();
    }
    // Each lane divides for one row, and the rows' scales go round.
    uint32_t mine = m[0];
    if (kBlock == 1) {
#pragma unroll
      for (int i = 1; i < U; ++i) mine = (sub & 3) == i ? m[i] : mine;
    }
    const float my_scale = __fdiv_rn(__uint_as_float(mine), kMax);
    const float my_recip = __fdiv_rn(1.0f, my_scale == 0.0f ? 1.0f : my_scale);
    if (kBlock == 1 ? sub < U && sub * kAcross < rows : threadIdx.x == 0)
      scales[kBlock == 1 ? sub * (kAcross * p.scale_rs) : 0] = my_scale;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float scale = kBlock == 1 ? __shfl_sync(0xffffffffu, my_scale, i, 4) : my_scale;
      const float recip = kBlock == 1 ? __shfl_sync(0xffffffffu, my_recip, i, 4) : my_recip;
      const Divisor by(scale, recip);
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        uint64_t f[4];
        v[i][j].get(f);
        by.template divide<sizeof(T) == 2 ? 1 : 2>(f);
        const int n = i * kAcross < rows ? cols - j * 8 * kLanes : 0;  // of eight channels, in range
        const uint32_t lo = e4m3x4(f[0], f[1]), hi = e4m3x4(f[2], f[3]);
        uint8_t* to = q + i * (kAcross * p.q_rs) + j * (8 * kLanes * q_cs);
        if (kWide) {
          if (n > 0) *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < n) to[e * kStep * q_cs] = uint8_t((e < 4 ? lo : hi) >> (8 * (e & 3)));
        }
      }
    }
  }
}

template <typename T, int kBlock, int kLanes, int U, bool kWide, bool kUnit>
cudaError_t launch_as(QuantParams p, cudaStream_t s) {
  p.row_blocks = cdiv64(p.T, kBlock == 1 ? 256 / kLanes * U : 128);
  const dim3 grid(unsigned(cdiv64(p.D, 128)), unsigned(std::min<int64_t>(p.row_blocks, 65535)));
  return launch(cconv_quantize_kernel<T, kBlock, kLanes, U, kWide, kUnit>, grid, kBlock == 1 ? 256 : 512, 0, 1, s, p);
}

template <typename T>
cudaError_t launch(const QuantParams& p, int block_rows, int sms, cudaStream_t s) {
  const uintptr_t in = reinterpret_cast<uintptr_t>(p.x) | uintptr_t(p.x_rs * int64_t(sizeof(T)));
  const uintptr_t out = reinterpret_cast<uintptr_t>(p.q) | uintptr_t(p.q_rs);
  const bool wide = sizeof(T) == 2 && p.D % 8 == 0 && p.x_cs == 1 && p.q_cs == 1 && (in & 15) == 0 && (out & 7) == 0;
  if constexpr (sizeof(T) == 2) {
    if (wide && block_rows == 128) return launch_as<T, 128, 16, 4, true, true>(p, s);
    // two rows a lane where that still fills the SMs (loads on their way cover HBM's latency), else one
    if (wide && cdiv64(p.T, 64) * cdiv64(p.D, 128) >= 4 * sms) return launch_as<T, 1, 8, 2, true, true>(p, s);
    if (wide) return launch_as<T, 1, 16, 1, true, true>(p, s);
  }
  if (p.x_cs == 1 && p.q_cs == 1) {  // (rows of an odd length: no multiplications for their addresses)
    if (block_rows == 128) return launch_as<T, 128, 16, 4, false, true>(p, s);
    return launch_as<T, 1, 16, 1, false, true>(p, s);
  }
  if (block_rows == 128) return launch_as<T, 128, 16, 4, false, false>(p, s);
  return launch_as<T, 1, 16, 1, false, false>(p, s);
}

}  // namespace

cudaError_t run_quantize(const QuantParams& p, int dtype, int block_rows, int sms, cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16) return launch<__nv_bfloat16>(p, block_rows, sms, s);
  if (dtype == CCONV_TYPE_FP16) return launch<__half>(p, block_rows, sms, s);
  return launch<float>(p, block_rows, sms, s);
}

}  // namespace cconv
