// Device helpers shared by the kernels of the feed-forward sub-block: element types and activations.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/cconv_block.h"

namespace cconv {
namespace {

__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(float v) { return v; }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }

// Every kernel of the sub-block is launched so that it may start while the kernel in front of it on its
// stream still runs, and begins with this: it touches memory only once that kernel is complete (which had
// waited for the one before it), and lets the next one be put in place.
__device__ __forceinline__ void start_in_order() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Two neighbouring elements of a 16-bit type as one 32-bit word (the first in the low half).
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// The activation's value a(g) and, if asked for, its derivative.  The exponential and the quotient are fast ones,
// whose error is relative and grows with the exponential's argument z (g, g^2/2, or gelu_tanh's 2z): s, Phi and so
// a(g) are within 2^-23 (16 + 4 |z|) of themselves in their tails too, 2e-6 at |z| = 0 and 4e-5 at 87, from where
// on they are 0 (an fp16 rounding: 5e-4, bf16: 4e-3).
//   silu       g s(g)              s(1 + g(1 - s)),          s = 1/(1 + exp(-g))
//   gelu       g Phi(g)            Phi + g exp(-g^2/2)/sqrt(2 pi)
//   gelu_tanh  g s(2z)             s + g s(1 - s) 2z',       z = sqrt(2/pi)(g + 0.044715 g^3)
//   relu       max(g, 0)           g > 0
template <int kAct, bool kDerivative>
__device__ __forceinline__ float activation_of(float g, float& da) {
  if constexpr (kAct == CCONV_ACT_SILU) {
    const float s = __fdividef(1.0f, 1.0f + __expf(-g));
    if (kDerivative) da = s * (1.0f + g * (1.0f - s));
    return g * s;
  } else if constexpr (kAct == CCONV_ACT_GELU) {
    // Phi(-x) = exp(-x^2/2) t P(t), t = 1 / (1 + 0.305 x), x = |g|: P of degree 7 is the one whose largest relative
    // error for x of 0 to 14 is least (1e-7; 4e-7 evaluated in 32 bits), fitted to erfcx(x / sqrt 2) / 2 by weighted
    // least squares (Lawson 1961).  Its exponential is the derivative's.
    const float e = __expf(-0.5f * g * g), t = __fdividef(1.0f, 1.0f + 0.305f * fabsf(g));
    const float poly = 0.1216397360f + t * (0.1224668175f + t * (0.1034208834f + t * (0.1210216209f + t * (-0.0379767232f +
                       t * (0.1857167780f + t * (-0.1529882550f + t * 0.0366991796f))))));
    const float tail = t * poly * e;  // Phi(-|g|)
    const float phi = g > 0.0f ? 1.0f - tail : tail;
    if (kDerivative) da = phi + g * 0.39894228040143268f * e;
    return g * phi;
  } else if constexpr (kAct == CCONV_ACT_GELU_TANH) {
    const float k = 1.5957691216057308f;  // 2 sqrt(2/pi)
    const float g2 = fminf(g * g, 1e12f);  // s is 0 or 1 long before: no infinity that s (1 - s) = 0 would multiply
    const float s = __fdividef(1.0f, 1.0f + __expf(-k * (g + 0.044715f * g * g2)));
    if (kDerivative) da = s + g * s * (1.0f - s) * k * (1.0f + 0.134145f * g2);
    return g * s;
  } else {
    if (kDerivative) da = g > 0.0f ? 1.0f : 0.0f;
    return g > 0.0f ? g : (g != g ? g : 0.0f);
  }
}
// h = a(g) u for N elements, in the place of g.  The choice is made once, not for each element: unrolled code
// for all four would not fit the instruction cache.
template <int kAct, int N>
__device__ __forceinline__ void gate_as(float (&g)[N], const float (&u)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float unused;
    g[i] = activation_of<kAct, false>(g[i], unused) * u[i];
  }
}
template <int N>
__device__ __forceinline__ void gate(int act, float (&g)[N], const float (&u)[N]) {
  if (act == CCONV_ACT_SILU) gate_as<CCONV_ACT_SILU>(g, u);
  else if (act == CCONV_ACT_GELU) gate_as<CCONV_ACT_GELU>(g, u);
  else if (act == CCONV_ACT_GELU_TANH) gate_as<CCONV_ACT_GELU_TANH>(g, u);
  else gate_as<CCONV_ACT_RELU>(g, u);
}
// From d = dL/dh, g and u: dL/dg in the place of g, dL/du in the place of d, h in the place of u.
template <int kAct, int N>
__device__ __forceinline__ void gate_backward_as(float (&d)[N], float (&g)[N], float (&u)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float da;
    const float a = activation_of<kAct, true>(g[i], da);
    g[i] = d[i] * u[i] * da;
    d[i] = d[i] * a;
    u[i] = a * u[i];
  }
}
template <int N>
__device__ __forceinline__ void gate_backward(int act, float (&d)[N], float (&g)[N], float (&u)[N]) {
  if (act == CCONV_ACT_SILU) gate_backward_as<CCONV_ACT_SILU>(d, g, u);
  else if (act == CCONV_ACT_GELU) gate_backward_as<CCONV_ACT_GELU>(d, g, u);
  else if (act == CCONV_ACT_GELU_TANH) gate_backward_as<CCONV_ACT_GELU_TANH>(d, g, u);
  else gate_backward_as<CCONV_ACT_RELU>(d, g, u);
}

// Pairs of fp32 values in a 64-bit register: two operations in one instruction.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ float2 halves_of(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

// Sum over the 32 lanes, the same in every lane.
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace
}  // namespace cconv
