// Products of at most 16 tokens: the weights are read once, straight into the registers that multiply them.
//
// What bounds them is HBM (a token costs 2 flops a weight), so the kernels are made of loads in flight: a
// tile is 16 rows of weights (8 of each matrix of the gated pair, or 8 of one where 16 would leave SMs
// idle), k is split over the 8 warps of a block, and a block goes through its tiles with the next 8 loads of
// 16 bytes of every lane on their way while the last 8 are multiplied, also across tiles.  The
// products run on warp-wide matrix instructions (m16n8: 16 rows of weights by 8 tokens) because they
// take operands from registers as they come from memory; tcgen05 would want them in shared memory first, for
// tiles that a few tokens leave almost empty.  Measured: one token 2048 x 8192 16 bits 23.2 us for 100.7 MB, 4.35 TB/s
// (a kernel that only reads as much, from as many threads: 18.4 to 20.7 us); two tokens 8192 x 4096 8 bits 10.2 us
// (reading alone: 8.2 us).  9 to 16 tokens take two such instructions a step (kEights = 2): 2048 x 8192 30 us and 512 x
// 1408 5.3, on pairs of CTAs 39 and 15; 8 bits 4096 x 4096 9.0, on pairs 14.4, and 8192 x 4096 16 on both.
//
// k is permuted inside a step: lane q of a row holds 16 neighbouring bytes of k, which stand for two
// pairs of fragment registers.  Weights and tokens are permuted alike, so the sums are those of the definition.
#include "block_few.h"

#include <algorithm>
#include <type_traits>

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
  int64_t x_lo;                   // bytes from a token's row to the row of what its rounding left (0: none)
  int64_t k_bytes, N;
  int T, act, weights_there;
  Mat out, out_lo, gate_pre, up_pre;
  const float *sa, *sb;
  int64_t sa_rs, sa_ks, sb_rs, sb_ks;
  int out_dtype;
};

// The sum of the block's warps for element (row r, token t) of a 16 x 8 tile, of which each wrote accumulator i of
// lane l at [i * 32 + l].
__device__ __forceinline__ float gathered(float (*smem)[128], int r, int t) {
  const int at = ((r >> 3) * 2 + (t & 1)) * 32 + (r & 7) * 4 + (t >> 1);
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

// The rows of a tile: 8 of w0 and the same 8 of w1, 16 of w0, or 8 of w0.
enum Rows { kPair, kSixteen, kEight };

// A block's tiles are blockIdx.x, blockIdx.x + gridDim.x, ...; every warp takes the same number of batches of
// each.  A step is 64 bytes of k a row (32 elements of 16 bits, or 64 of 8, two of which make a block that
// shares a scale); a batch is 8 loads a lane.
template <typename T, Rows kRows, int kEights>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_few_kernel(const FewParams p) {
  __shared__ float smem[2][kEights][kWarps][128];
  constexpr bool kFp8 = std::is_same<T, E4m3>::value;
  constexpr int kSteps = kRows == kEight ? 8 : 4, kHalf = kRows == kEight ? 1 : 2;
  constexpr int kTile = kRows == kSixteen ? 16 : 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int tiles = int((p.N + kTile - 1) / kTile);
  const int steps = int((p.k_bytes + 63) / 64), unit = kFp8 ? 2 : 1;
  const int per = ((steps + unit - 1) / unit + kWarps - 1) / kWarps * unit;  // steps of a warp
  const int s0 = warp * per, s1 = min(steps, s0 + per), batches = (per + kSteps - 1) / kSteps;
  const int mine = int(blockIdx.x) < tiles ? (tiles - 1 - int(blockIdx.x)) / int(gridDim.x) + 1 : 0;
  const uint4 none = make_uint4(0, 0, 0, 0);
  uint4 w[2][8];

  // where the next batch comes from
  int lt = blockIdx.x, lb = 0;
  auto load = [&](uint4 (&a)[8]) {
    if (lt < tiles) {
      const int64_t r = int64_t(lt) * kTile + g, last = p.N - 1;
      const char* w0 = p.w0 + min(r, last) * p.w0_rs + q * 16;
      const char* w1 = kRows == kPair ? p.w1 + min(r, last) * p.w1_rs + q * 16 : p.w0 + min(r + 8, last) * p.w0_rs + q * 16;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int s = s0 + lb * kSteps + i;
        const int64_t at = int64_t(s) * 64;
        const bool in = s < s1 && at + q * 16 < p.k_bytes;
        a[i * kHalf] = in ? load_weights(w0 + at) : none;
        if (kHalf == 2) a[i * 2 + 1] = in ? load_weights(w1 + at) : none;
      }
    }
    if (++lb == batches) lb = 0, lt += gridDim.x;
  };

  // Behind this kernel's other form in the same call, which lets it in only once everything before the call is
  // complete, the weights are there already, and only the tokens may still be on their way.
  if (p.weights_there) load(w[0]);
  start_in_order();
  if (!p.weights_there) load(w[0]);

  // Column g of a tile is token g; tokens in two parts (at most 4) take columns g and g + 4.
  const bool parts = !kFp8 && kRows != kPair && kEights == 1 && p.x_lo != 0;
  float acc[kEights][4] = {};
  int tile = blockIdx.x, batch = 0, parity = 0;
  auto use = [&](const uint4 (&a)[8]) {
    const int sb = s0 + batch * kSteps;
#pragma unroll
    for (int e = 0; e < kEights; ++e) {
      const int token = parts ? g & 3 : g + 8 * e;
      const char* const x = p.x + min(token, p.T - 1) * p.x_rs + (parts && g >= 4 ? p.x_lo : 0) + q * 16;
      uint4 v[kSteps];
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int64_t at = int64_t(sb + i) * 64;
        v[i] = token < p.T && sb + i < s1 && at + q * 16 < p.k_bytes ? load_tokens(x + at) : none;
      }
      if constexpr (!kFp8) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const uint4 a0 = a[i * kHalf], a1 = kHalf == 2 ? a[i * kHalf + kHalf - 1] : none;
          mma<T>(acc[e], a0.x, a1.x, a0.y, a1.y, v[i].x, v[i].y);
          mma<T>(acc[e], a0.z, a1.z, a0.w, a1.w, v[i].z, v[i].w);
        }
      } else {
        // the sums of a block of 128 are scaled before they are added up; the rows of a tile share their scale
        const int64_t nb = int64_t(tile) * kTile >> 7;
        const int t0 = min(8 * e + 2 * q, p.T - 1), t1 = min(8 * e + 2 * q + 1, p.T - 1);  // whose sums this lane holds
#pragma unroll
        for (int j = 0; j < kSteps / 2; ++j) {
          if (sb + 2 * j < s1) {
            const int64_t kb = (sb >> 1) + j;
            const float s = p.sb[nb * p.sb_rs + kb * p.sb_ks];
            const float sa0 = s * p.sa[t0 * p.sa_rs + kb * p.sa_ks], sa1 = s * p.sa[t1 * p.sa_rs + kb * p.sa_ks];
            float d[4] = {};
#pragma unroll
            for (int i = 2 * j; i < 2 * j + 2; ++i) {
              const uint4 a0 = a[i * kHalf], a1 = kHalf == 2 ? a[i * kHalf + kHalf - 1] : none;
              mma<T>(d, a0.x, a1.x, a0.y, a1.y, v[i].x, v[i].y);
              mma<T>(d, a0.z, a1.z, a0.w, a1.w, v[i].z, v[i].w);
            }
            acc[e][0] += sa0 * d[0];
            acc[e][1] += sa1 * d[1];
            acc[e][2] += sa0 * d[2];
            acc[e][3] += sa1 * d[3];
          }
        }
      }
    }
    if (++batch < batches) return;
    batch = 0;
#pragma unroll
    for (int e = 0; e < kEights; ++e) {
#pragma unroll
      for (int i = 0; i < 4; ++i) smem[parity][e][warp][i * 32 + lane] = acc[e][i], acc[e][i] = 0.0f;
    }
    __syncthreads();
    const int64_t n0 = int64_t(tile) * kTile;
    const int r = threadIdx.x % kTile, t = threadIdx.x / kTile;
    if (t < p.T && n0 + r < p.N) {
      float f = gathered(smem[parity][t >> 3 & (kEights - 1)], r, t & 7);
      if (parts) f += gathered(smem[parity][0], r, t + 4);
      if constexpr (kRows == kPair) {
        const float up = gathered(smem[parity][t >> 3 & (kEights - 1)], r + 8, t & 7);
        float h[1] = {f};
        const float u[1] = {up};
        gate(p.act, h, u);
        // in two parts, whose sum has the type's precision twice (what overflows has no second part)
        const T hi = from_f32<T>(h[0]);
        put(p.out, p.out_dtype, t, n0 + r, to_f32(hi));
        if (p.out_lo.p) put(p.out_lo, p.out_dtype, t, n0 + r, isfinite(to_f32(hi)) ? h[0] - to_f32(hi) : 0.0f);
        if (p.gate_pre.p) {
          put(p.gate_pre, p.out_dtype, t, n0 + r, f);
          put(p.up_pre, p.out_dtype, t, n0 + r, up);
        }
      } else {
        put(p.out, p.out_dtype, t, n0 + r, f);
      }
    }
    parity ^= 1;
    tile += gridDim.x;
  };
  const int total = mine * batches;
  for (int it = 0; it < total; it += 2) {
    load(w[1]);
    use(w[0]);
    if (it + 1 < total) {
      load(w[0]);
      use(w[1]);
    }
  }
}

template <typename T, Rows kRows, int kEights>
cudaError_t launch_eights(const FewParams& p, int sms, cudaStream_t s) {
  const int64_t tiles = cdiv64(p.N, kRows == kSixteen ? 16 : 8);
  const dim3 grid(unsigned(std::min<int64_t>(tiles, 2 * sms)));
  return launch(cconv_few_kernel<T, kRows, kEights>, grid, kWarps * 32, 0, 1, s, p);
}
template <typename T, Rows kRows>
cudaError_t launch_rows(const FewParams& p, int sms, cudaStream_t s) {
  if (p.T > 8) return launch_eights<T, kRows, 2>(p, sms, s);
  return launch_eights<T, kRows, 1>(p, sms, s);
}

// 16 rows a tile where that leaves no SM idle: one token, 16 bits, the product back to 4096 channels as part of
// 4096 x 8192 whole: 37 against 41 us; to 2048 channels 8 rows a tile are better (2048 x 8192 whole: 23.7 against
// 25.4 us).
template <typename T>
cudaError_t launch_single(const FewParams& p, int sms, cudaStream_t s) {
  return p.N >= 16 * int64_t(sms) ? launch_rows<T, kSixteen>(p, sms, s) : launch_rows<T, kEight>(p, sms, s);
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
                          const Mat& h, const Mat& h_lo, int64_t T, int64_t F, int64_t D, int act, int dtype, int sms,
                          cudaStream_t s) {
  FewParams p = params(x, wg, h, T, F, D, 2, dtype);
  p.w1 = static_cast<const char*>(wu.p);
  p.w1_rs = wu.rs * 2;
  p.out_lo = h_lo;
  p.gate_pre = gate_pre;
  p.up_pre = up_pre;
  p.act = act;
  return dtype == CCONV_TYPE_BF16 ? launch_rows<__nv_bfloat16, kPair>(p, sms, s)
                                  : launch_rows<__half, kPair>(p, sms, s);
}

cudaError_t run_few_product(const Mat& x, const Mat& x_lo, const Mat& w, const Mat& out, int64_t T, int64_t N,
                            int64_t K, int dtype, int sms, bool weights_there, cudaStream_t s) {
  FewParams p = params(x, w, out, T, N, K, 2, dtype);
  p.weights_there = weights_there;
  if (x_lo.p) p.x_lo = static_cast<const char*>(x_lo.p) - p.x;
  return dtype == CCONV_TYPE_BF16 ? launch_single<__nv_bfloat16>(p, sms, s)
                                  : launch_single<__half>(p, sms, s);
}

cudaError_t run_few_fp8(const Mat& x, const Mat& w, const Mat& sa, const Mat& sb, const Mat& out, int64_t T, int64_t N,
                        int64_t K, int dtype, int sms, cudaStream_t s) {
  FewParams p = params(x, w, out, T, N, K, 1, dtype);
  p.sa = static_cast<const float*>(sa.p);
  p.sa_rs = sa.rs;
  p.sa_ks = sa.cs;
  p.sb = static_cast<const float*>(sb.p);
  p.sb_rs = sb.rs;
  p.sb_ks = sb.cs;
  // 8 rows a tile take twice the scales a row: 4096 x 4096 8.7 against 6.2 us, 4096 x 1024 5.3 against 2.9, 1024 x
  // 1024 2.6 against 2.1; they win only where rows are few and long (1024 x 8192: 6.4 against 7.3)
  return launch_rows<E4m3, kSixteen>(p, sms, s);
}

}  // namespace cconv
