// Products of the feed-forward block.
#include <cuda_fp8.h>

#include "block.h"
#include "block_device.cuh"
#include "block_gemm.h"

namespace cconv {
namespace {

__device__ __forceinline__ float to_f32(__nv_fp8_e4m3 v) { return float(v); }

// 64 x 64 outputs a block of 256 threads, 4 x 4 a thread; k in steps of 16 through shared memory.
// fp8: sums of 128 products are scaled before they are added up.
template <typename T, typename Out, bool kFp8>
__global__ void __launch_bounds__(256) cconv_product_kernel(Mat a, Mat b, Mat sa, Mat sb, Mat c, int64_t M,
                                                            int64_t N, int64_t K, int add) {
  __shared__ float as[16][65], bs[16][65];
  const int64_t m0 = int64_t(blockIdx.y) * 64, n0 = int64_t(blockIdx.x) * 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const T* A = static_cast<const T*>(a.p);
  const T* B = static_cast<const T*>(b.p);
  float total[4][4] = {}, acc[4][4] = {};
  for (int64_t k0 = 0; k0 < K; k0 += 16) {
    for (int i = threadIdx.x; i < 1024; i += 256) {
      const int k = i & 15, r = i >> 4;
      as[k][r] = m0 + r < M && k0 + k < K ? to_f32(A[(m0 + r) * a.rs + (k0 + k) * a.cs]) : 0.0f;
      bs[k][r] = n0 + r < N && k0 + k < K ? to_f32(B[(n0 + r) * b.rs + (k0 + k) * b.cs]) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += as[k][ty * 4 + i] * bs[k][tx * 4 + j];
    __syncthreads();
    if (kFp8 && ((k0 + 16) % 128 == 0 || k0 + 16 >= K)) {
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
          const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j, kb = k0 / 128;
          if (m < M && n < N)
            total[i][j] += acc[i][j] * (static_cast<const float*>(sa.p)[m * sa.rs + kb * sa.cs] *
                                        static_cast<const float*>(sb.p)[n / 128 * sb.rs + kb * sb.cs]);
          acc[i][j] = 0.0f;
        }
    }
  }
  Out* C = static_cast<Out*>(const_cast<void*>(c.p));
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m >= M || n >= N) continue;
      float v = kFp8 ? total[i][j] : acc[i][j];
      Out* to = C + m * c.rs + n * c.cs;
      if (add) v += cconv::to_f32(*to);
      *to = from_f32<Out>(v);
    }
}

// Finishing passes over the sums: 256 threads a block along n, a row a blockIdx.y step.
template <typename T>
__global__ void __launch_bounds__(256) finish_store_kernel(const float* sums, Mat out, int64_t M, int64_t N) {
  const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (n >= N) return;
  T* o = static_cast<T*>(const_cast<void*>(out.p));
  for (int64_t m = blockIdx.y; m < M; m += gridDim.y) o[m * out.rs + n * out.cs] = from_f32<T>(sums[m * N + n]);
}

template <typename T>
__global__ void __launch_bounds__(256) finish_gated_kernel(const float* g, const float* u, Mat gate_pre, Mat up_pre,
                                                           Mat h, int64_t M, int64_t N, int act) {
  const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (n >= N) return;
  for (int64_t m = blockIdx.y; m < M; m += gridDim.y) {
    float da;
    const float gv = g[m * N + n], uv = u[m * N + n];
    static_cast<T*>(const_cast<void*>(h.p))[m * h.rs + n * h.cs] = from_f32<T>(activation<false>(act, gv, da) * uv);
    if (gate_pre.p) {
      static_cast<T*>(const_cast<void*>(gate_pre.p))[m * gate_pre.rs + n * gate_pre.cs] = from_f32<T>(gv);
      static_cast<T*>(const_cast<void*>(up_pre.p))[m * up_pre.rs + n * up_pre.cs] = from_f32<T>(uv);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) finish_gated_backward_kernel(const float* dh, Mat gate_pre, Mat up_pre,
                                                                    Mat dg, Mat du, Mat h, int64_t M, int64_t N,
                                                                    int act) {
  const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (n >= N) return;
  for (int64_t m = blockIdx.y; m < M; m += gridDim.y) {
    const float g = to_f32(static_cast<const T*>(gate_pre.p)[m * gate_pre.rs + n * gate_pre.cs]);
    const float u = to_f32(static_cast<const T*>(up_pre.p)[m * up_pre.rs + n * up_pre.cs]);
    const float d = dh[m * N + n];
    float da;
    const float a = activation<true>(act, g, da);
    static_cast<T*>(const_cast<void*>(dg.p))[m * dg.rs + n * dg.cs] = from_f32<T>(d * u * da);
    static_cast<T*>(const_cast<void*>(du.p))[m * du.rs + n * du.cs] = from_f32<T>(d * a);
    static_cast<T*>(const_cast<void*>(h.p))[m * h.rs + n * h.cs] = from_f32<T>(a * u);
  }
}

dim3 product_grid(int64_t M, int64_t N) { return dim3(unsigned(cdiv64(N, 64)), unsigned(cdiv64(M, 64))); }
dim3 finish_grid(int64_t M, int64_t N) { return dim3(unsigned(cdiv64(N, 256)), unsigned(M < 16384 ? M : 16384)); }

}  // namespace

cudaError_t run_product_simple(const Mat& a, const Mat& b, float* c, int64_t M, int64_t N, int64_t K, int dtype,
                               bool add, cudaStream_t s) {
  const Mat cm(c, N, 1), none;
  if (dtype == CCONV_TYPE_BF16)
    cconv_product_kernel<__nv_bfloat16, float, false><<<product_grid(M, N), 256, 0, s>>>(a, b, none, none, cm, M, N, K, add);
  else
    cconv_product_kernel<__half, float, false><<<product_grid(M, N), 256, 0, s>>>(a, b, none, none, cm, M, N, K, add);
  return cudaGetLastError();
}

cudaError_t run_fp8_simple(const Mat& a, const Mat& b, const Mat& sa, const Mat& sb, const Mat& c, int64_t M,
                           int64_t N, int64_t K, int dtype, cudaStream_t s) {
  using E = __nv_fp8_e4m3;
  const dim3 grid = product_grid(M, N);
  if (dtype == CCONV_TYPE_BF16)
    cconv_product_kernel<E, __nv_bfloat16, true><<<grid, 256, 0, s>>>(a, b, sa, sb, c, M, N, K, 0);
  else if (dtype == CCONV_TYPE_FP16)
    cconv_product_kernel<E, __half, true><<<grid, 256, 0, s>>>(a, b, sa, sb, c, M, N, K, 0);
  else
    cconv_product_kernel<E, float, true><<<grid, 256, 0, s>>>(a, b, sa, sb, c, M, N, K, 0);
  return cudaGetLastError();
}

cudaError_t finish_store(const float* sums, const Mat& out, int64_t M, int64_t N, int dtype, cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16) finish_store_kernel<__nv_bfloat16><<<finish_grid(M, N), 256, 0, s>>>(sums, out, M, N);
  else finish_store_kernel<__half><<<finish_grid(M, N), 256, 0, s>>>(sums, out, M, N);
  return cudaGetLastError();
}

cudaError_t finish_gated(const float* g, const float* u, const Mat& gate_pre, const Mat& up_pre, const Mat& h,
                         int64_t M, int64_t N, int act, int dtype, cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16)
    finish_gated_kernel<__nv_bfloat16><<<finish_grid(M, N), 256, 0, s>>>(g, u, gate_pre, up_pre, h, M, N, act);
  else
    finish_gated_kernel<__half><<<finish_grid(M, N), 256, 0, s>>>(g, u, gate_pre, up_pre, h, M, N, act);
  return cudaGetLastError();
}

cudaError_t finish_gated_backward(const float* dh, const Mat& gate_pre, const Mat& up_pre, const Mat& dg,
                                  const Mat& du, const Mat& h, int64_t M, int64_t N, int act, int dtype,
                                  cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16)
    finish_gated_backward_kernel<__nv_bfloat16><<<finish_grid(M, N), 256, 0, s>>>(dh, gate_pre, up_pre, dg, du, h, M, N, act);
  else
    finish_gated_backward_kernel<__half><<<finish_grid(M, N), 256, 0, s>>>(dh, gate_pre, up_pre, dg, du, h, M, N, act);
  return cudaGetLastError();
}

}  // namespace cconv
