// Products of at most 16 tokens: the weights are read once, straight into the registers that multiply them.
//
// What bounds them is HBM (a token costs 2 flops a weight), so the kernels are made of loads in flight: a
// block takes 16 rows of weights (8 of each matrix of the gated pair) and splits k over its 8 warps, every
// lane has 16 loads of 16 bytes on their way, and all blocks of a served layer are resident at once.  The
// products run on warp-wide matrix instructions (m16n8: 16 rows of weights by 8 tokens) because they
// take operands from registers as they come from memory; tcgen05 would want them in shared memory first, for
// tiles that a few tokens leave almost empty.
//
// k is permuted inside a step: lane q of a row holds 16 neighbouring bytes of k, which stand for two
// pairs of fragment registers.  Weights and tokens are permuted alike, so the sums are those of the definition.
#include "block_few.h"

#include <algorithm>

#include "block_device.cuh"
#include "block_launch.h"

namespace cconv {
namespace {

constexpr int kWarps = 8;

template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
struct E4m3 {};
template <>
__device__ __forceinline__ void mma<E4m3>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Weights pass by once: not kept in L1, which the tokens share.
__device__ __forceinline__ uint4 load_weights(const char* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint4 load_tokens(const char* p) { return *reinterpret_cast<const uint4*>(p); }

struct FewParams {
  const char *x, *w0, *w1;        // tokens; weights (w1: the second matrix of a pair)
  int64_t x_rs, w0_rs, w1_rs;     // bytes
  int64_t k_bytes, N;
  int T, act, more;
  Mat out, gate_pre, up_pre;
  const float *sa, *sb;
  int64_t sa_rs, sa_ks, sb_rs, sb_ks;
  int out_dtype;
};

// Sums of the block's warps: element (row r, token t) of the 16 x 8 B tile.
template <int B>
__device__ __forceinline__ void gather(float (*smem)[B * 128], const float (&acc)[B][4], int warp, int lane) {
#pragma unroll
  for (int b = 0; b < B; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) smem[warp][b * 128 + i * 32 + lane] = acc[b][i];
  __syncthreads();
}
template <int B>
__device__ __forceinline__ float gathered(float (*smem)[B * 128], int r, int t) {
  const int at = (t >> 3) * 128 + ((r >> 3) * 2 + (t & 1)) * 32 + (r & 7) * 4 + ((t & 7) >> 1);
  float s = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s += smem[w][at];
  return s;
}

__device__ __forceinline__ void put(const Mat& m, int dtype, int64_t r, int64_t c, float v) {
  const int64_t at = r * m.rs + c * m.cs;
  char* p = static_cast<char*>(const_cast<void*>(m.p));
  if (dtype == CCONV_TYPE_BF16) reinterpret_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
  else if (dtype == CCONV_TYPE_FP16) reinterpret_cast<__half*>(p)[at] = __float2half_rn(v);
  else reinterpret_cast<float*>(p)[at] = v;
}

// 16-bit types.  kPair: rows 0-7 of the tile are 8 rows of w0, rows 8-15 the same rows of w1, else 16 rows of w0.
// B: blocks of 8 tokens.  A step is 64 bytes of k a row (32 elements).
template <typename T, bool kPair, int B>
__global__ void __launch_bounds__(kWarps * 32) cconv_few_kernel(const FewParams p) {
  __shared__ float smem[kWarps][B * 128];
  constexpr int kSteps = 8;  // loaded together
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int64_t n0 = int64_t(blockIdx.x) * (kPair ? 8 : 16), last = p.N - 1;
  const char* w0 = p.w0 + min(n0 + g, last) * p.w0_rs + q * 16;
  const char* w1 = kPair ? p.w1 + min(n0 + g, last) * p.w1_rs + q * 16 : p.w0 + min(n0 + 8 + g, last) * p.w0_rs + q * 16;
  const int64_t steps = (p.k_bytes + 63) / 64, per = (steps + kWarps - 1) / kWarps;
  const int64_t s0 = warp * per, s1 = min(steps, s0 + per);
  float acc[B][4] = {};
  const uint4 none = make_uint4(0, 0, 0, 0);
  bool waited = false;
  for (int64_t s = s0; s < s1 || !waited; s += kSteps) {
    uint4 a[kSteps], c[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int64_t at = (s + i) * 64;
      const bool in = s + i < s1 && at + q * 16 < p.k_bytes;
      a[i] = in ? load_weights(w0 + at) : none;
      c[i] = in ? load_weights(w1 + at) : none;
    }
    if (!waited) {
      // the weights were there before this call; the tokens may come from the kernel in front
      asm volatile("griddepcontrol.wait;" ::: "memory");
      if (p.more) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
      waited = true;
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int t = b * 8 + g;
      const char* x = p.x + min(t, p.T - 1) * p.x_rs + q * 16;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int64_t at = (s + i) * 64;
        const uint4 v = t < p.T && s + i < s1 && at + q * 16 < p.k_bytes ? load_tokens(x + at) : none;
        mma<T>(acc[b], a[i].x, c[i].x, a[i].y, c[i].y, v.x, v.y);
        mma<T>(acc[b], a[i].z, c[i].z, a[i].w, c[i].w, v.z, v.w);
      }
    }
  }
  gather<B>(smem, acc, warp, lane);
  const int dtype = sizeof(T) == 2 && p.out_dtype == CCONV_TYPE_BF16 ? CCONV_TYPE_BF16 : CCONV_TYPE_FP16;
  if (kPair) {
    const int r = threadIdx.x & 7, t = threadIdx.x >> 3;
    if (t < p.T && t < 8 * B && n0 + r < p.N) {
      const float gate = gathered<B>(smem, r, t), up = gathered<B>(smem, r + 8, t);
      float unused;
      put(p.out, dtype, t, n0 + r, activation<false>(p.act, gate, unused) * up);
      if (p.gate_pre.p) {
        put(p.gate_pre, dtype, t, n0 + r, gate);
        put(p.up_pre, dtype, t, n0 + r, up);
      }
    }
  } else {
    const int r = threadIdx.x & 15, t = threadIdx.x >> 4;
    if (t < p.T && t < 8 * B && n0 + r < p.N) put(p.out, dtype, t, n0 + r, gathered<B>(smem, r, t));
  }
}

// 8-bit operands: a step is 64 bytes = 64 elements of k a row, two steps a block of 128, whose sums are
// scaled before they are added up.  The 16 rows share their scale.
template <int B>
__global__ void __launch_bounds__(kWarps * 32) cconv_few_fp8_kernel(const FewParams p) {
  __shared__ float smem[kWarps][B * 128];
  constexpr int kBlocks = 4;  // loaded together
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int64_t n0 = int64_t(blockIdx.x) * 16, last = p.N - 1;
  const char* w0 = p.w0 + min(n0 + g, last) * p.w0_rs + q * 16;
  const char* w1 = p.w0 + min(n0 + 8 + g, last) * p.w0_rs + q * 16;
  const float* sb = p.sb + (n0 >> 7) * p.sb_rs;
  const int64_t kbs = (p.k_bytes + 127) / 128, per = (kbs + kWarps - 1) / kWarps;
  const int64_t k0 = warp * per, k1 = min(kbs, k0 + per);
  float total[B][4] = {};
  const uint4 none = make_uint4(0, 0, 0, 0);
  for (int64_t kb = k0; kb < k1; kb += kBlocks) {
    uint4 a[2 * kBlocks], c[2 * kBlocks];
#pragma unroll
    for (int i = 0; i < 2 * kBlocks; ++i) {
      const int64_t at = kb * 128 + i * 64;
      const bool in = kb + i / 2 < k1 && at + q * 16 < p.k_bytes;
      a[i] = in ? load_weights(w0 + at) : none;
      c[i] = in ? load_weights(w1 + at) : none;
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int t = b * 8 + g;
      const char* x = p.x + min(t, p.T - 1) * p.x_rs + q * 16;
      const int t0 = b * 8 + 2 * q;  // the two tokens whose sums this lane holds
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        if (kb + j >= k1) break;
        float acc[4] = {};
#pragma unroll
        for (int i = 2 * j; i < 2 * j + 2; ++i) {
          const int64_t at = kb * 128 + i * 64;
          const uint4 v = t < p.T && at + q * 16 < p.k_bytes ? load_tokens(x + at) : none;
          mma<E4m3>(acc, a[i].x, c[i].x, a[i].y, c[i].y, v.x, v.y);
          mma<E4m3>(acc, a[i].z, c[i].z, a[i].w, c[i].w, v.z, v.w);
        }
        const float s = sb[(kb + j) * p.sb_ks];
        const float s0 = s * p.sa[min(t0, p.T - 1) * p.sa_rs + (kb + j) * p.sa_ks];
        const float s1 = s * p.sa[min(t0 + 1, p.T - 1) * p.sa_rs + (kb + j) * p.sa_ks];
        total[b][0] += s0 * acc[0];
        total[b][1] += s1 * acc[1];
        total[b][2] += s0 * acc[2];
        total[b][3] += s1 * acc[3];
      }
    }
  }
  gather<B>(smem, total, warp, lane);
  const int r = threadIdx.x & 15, t = threadIdx.x >> 4;
  if (t < p.T && t < 8 * B && n0 + r < p.N) put(p.out, p.out_dtype, t, n0 + r, gathered<B>(smem, r, t));
}

template <typename T, bool kPair>
cudaError_t launch_few(const FewParams& p, bool chained, cudaStream_t s) {
  const dim3 grid(unsigned(cdiv64(p.N, kPair ? 8 : 16)));
  return p.T <= 8 ? launch(cconv_few_kernel<T, kPair, 1>, grid, kWarps * 32, 0, 1, chained, s, p)
                  : launch(cconv_few_kernel<T, kPair, 2>, grid, kWarps * 32, 0, 1, chained, s, p);
}

FewParams params(const Mat& x, const Mat& w, const Mat& out, int64_t T, int64_t N, int64_t K, int es, int dtype) {
  FewParams p{};
  p.x = static_cast<const char*>(x.p);
  p.x_rs = x.rs * es;
  p.w0 = static_cast<const char*>(w.p);
  p.w0_rs = w.rs * es;
  p.k_bytes = K * es;
  p.N = N;
  p.T = int(T);
  p.out = out;
  p.out_dtype = dtype;
  return p;
}

}  // namespace

bool few_readable(const Mat& m, int64_t rows, int64_t k, int es) {
  const int64_t unit = 16 / es;
  return (reinterpret_cast<uintptr_t>(m.p) & 15u) == 0 && (m.cs == 1 || k == 1) && k % unit == 0 &&
         (rows == 1 || m.rs % unit == 0);
}

cudaError_t run_few_gated(const Mat& x, const Mat& wg, const Mat& wu, const Mat& gate_pre, const Mat& up_pre,
                          const Mat& h, int64_t T, int64_t F, int64_t D, int act, int dtype, bool more, cudaStream_t s) {
  FewParams p = params(x, wg, h, T, F, D, 2, dtype);
  p.w1 = static_cast<const char*>(wu.p);
  p.w1_rs = wu.rs * 2;
  p.gate_pre = gate_pre;
  p.up_pre = up_pre;
  p.act = act;
  p.more = more;
  return dtype == CCONV_TYPE_BF16 ? launch_few<__nv_bfloat16, true>(p, false, s) : launch_few<__half, true>(p, false, s);
}

cudaError_t run_few_product(const Mat& x, const Mat& w, const Mat& out, int64_t T, int64_t N, int64_t K, int dtype,
                            bool chained, bool more, cudaStream_t s) {
  FewParams p = params(x, w, out, T, N, K, 2, dtype);
  p.more = more;
  return dtype == CCONV_TYPE_BF16 ? launch_few<__nv_bfloat16, false>(p, chained, s)
                                  : launch_few<__half, false>(p, chained, s);
}

cudaError_t run_few_fp8(const Mat& x, const Mat& w, const Mat& sa, const Mat& sb, const Mat& out, int64_t T, int64_t N,
                        int64_t K, int dtype, cudaStream_t s) {
  FewParams p = params(x, w, out, T, N, K, 1, dtype);
  p.sa = static_cast<const float*>(sa.p);
  p.sa_rs = sa.rs;
  p.sa_ks = sa.cs;
  p.sb = static_cast<const float*>(sb.p);
  p.sb_rs = sb.rs;
  p.sb_ks = sb.cs;
  const dim3 grid(unsigned(cdiv64(N, 16)));
  return T <= 8 ? launch(cconv_few_fp8_kernel<1>, grid, kWarps * 32, 0, 1, false, s, p)
                : launch(cconv_few_fp8_kernel<2>, grid, kWarps * 32, 0, 1, false, s, p);
}

}  // namespace cconv
