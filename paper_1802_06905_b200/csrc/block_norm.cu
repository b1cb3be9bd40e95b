// Norms before and after a block, fused with the block's gate and the residual scale.
//
//   forward    n = y rho_y w_post,  r' = scale r + gate n,  x = r' rho_r w_pre,
//              rho_v = 1 / sqrt(mean(v^2) + eps)
//   backward   e = dx w_pre,  S = dr' + rho_r e - r' rho_r^3 mean(e r')       (dL/dr', all of it)
//              dr = scale S,  dgate = sum_t S n,  dn = gate S
//              f = dn w_post,  dy = rho_y f - y rho_y^3 mean(f y)
//              dw_post = sum_t dn y rho_y,  dw_pre = sum_t dx r' rho_r
//
// Both directions read every [T][D] array once and write every output once; a row stays in registers
// between its two reductions (over y, then over r'; backward: over r' and e, then over y and f), so
// they are bound by HBM.
#include <algorithm>

#include "block.h"
#include "block_device.cuh"
#include "block_norm.h"
#include "host_setup.h"

namespace cconv {
namespace {

// E elements of type T that are loaded and stored together.
template <typename T, int E>
struct Vec;
template <typename T>
struct Vec<T, 8> {  // 16-bit types
  uint4 w;
  __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { w = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y), c = unpack2<T>(w.z), d = unpack2<T>(w.w);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
  }
  static __device__ __forceinline__ void store(T* p, const float (&f)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]),
                                              pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
  }
};
template <>
struct Vec<float, 4> {
  float4 w;
  __device__ __forceinline__ void load(const float* p) { w = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void zero() { w = make_float4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = w.x; f[1] = w.y; f[2] = w.z; f[3] = w.w; }
  static __device__ __forceinline__ void store(float* p, const float (&f)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  }
};
template <typename T>
struct Vec<T, 1> {
  T w;
  __device__ __forceinline__ void load(const T* p) { w = *p; }
  __device__ __forceinline__ void zero() { w = from_f32<T>(0.0f); }
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f32(w); }
  static __device__ __forceinline__ void store(T* p, const float (&f)[1]) { *p = from_f32<T>(f[0]); }
};

// Sums of two values over the block, the same in every thread.  `buf` alternates between calls, so
// that one barrier a call is enough.
__device__ __forceinline__ float2 block_sum2(float a, float b, float2 (*smem)[32], int& buf) {
  a = warp_sum(a);
  b = warp_sum(b);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return make_float2(a, b);
  if ((threadIdx.x & 31) == 0) smem[buf][threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const float2 v = lane < warps ? smem[buf][lane] : make_float2(0.0f, 0.0f);
  buf ^= 1;
  return make_float2(warp_sum(v.x), warp_sum(v.y));
}

// ---- forward -----------------------------------------------------------------------------------
template <typename T, int E, int NV>
__global__ void __launch_bounds__(1024) cconv_residual_norm_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  using V = Vec<T, E>;
  const T* resid = static_cast<const T*>(p.resid);  // may be resid_out
  const T* __restrict__ block = static_cast<const T*>(p.block);
  const T* __restrict__ gate = static_cast<const T*>(p.gate);
  const T* __restrict__ w_post = static_cast<const T*>(p.w_post);
  const T* __restrict__ w_pre = static_cast<const T*>(p.w_pre);
  T* resid_out = static_cast<T*>(p.resid_out);
  T* norm_out = static_cast<T*>(p.norm_out);
  const int nt = blockDim.x, tid = threadIdx.x;
  const float inv_d = 1.0f / float(p.D);
  int buf = 0;
  V r[NV], y[NV];
  auto fetch = [&](int64_t t) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      r[v].zero();
      y[v].zero();
      if (c < p.D) {
        r[v].load(resid + t * p.resid_rs + c);
        if (block) y[v].load(block + t * p.block_rs + c);
      }
    }
  };
  int64_t t = blockIdx.x;
  if (t < p.T) fetch(t);
  for (; t < p.T; t += gridDim.x) {
    float o[NV][E], n[NV][E];
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      r[v].get(o[v]);
      y[v].get(n[v]);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        o[v][i] *= p.scale;
        ss += n[v][i] * n[v][i];
      }
    }
    // the next row of this block is on its way while this one is reduced
    if (t + gridDim.x < p.T) fetch(t + gridDim.x);
    if (block) {
      float rho = 1.0f;
      if (w_post) rho = rsqrtf(block_sum2(ss, 0.0f, smem, buf).x * inv_d + p.eps);
      const T* g = gate ? gate + (p.rows_per_gate ? t / p.rows_per_gate : 0) * p.gate_rs : nullptr;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * nt + tid) * E;
        if (c >= p.D) continue;
        float f[E];
        if (w_post) {
          V w;
          w.load(w_post + c);
          w.get(f);
#pragma unroll
          for (int i = 0; i < E; ++i) n[v][i] *= rho * f[i];
        }
        if (g) {
          V w;
          w.load(g + c);
          w.get(f);
#pragma unroll
          for (int i = 0; i < E; ++i) n[v][i] *= f[i];
        }
#pragma unroll
        for (int i = 0; i < E; ++i) o[v][i] += n[v][i];
      }
    }
    ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      if (c < p.D) V::store(resid_out + t * p.resid_out_rs + c, o[v]);
#pragma unroll
      for (int i = 0; i < E; ++i) ss += o[v][i] * o[v][i];
    }
    if (norm_out) {
      const float rho = rsqrtf(block_sum2(ss, 0.0f, smem, buf).x * inv_d + p.eps);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * nt + tid) * E;
        if (c >= p.D) continue;
        float f[E];
        if (w_pre) {
          V w;
          w.load(w_pre + c);
          w.get(f);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) o[v][i] *= w_pre ? rho * f[i] : rho;
        V::store(norm_out + t * p.norm_out_rs + c, o[v]);
      }
    }
  }
}

// Rows too long for registers: the row is read again in each of the three sweeps (from L2).
template <typename T>
__global__ void __launch_bounds__(1024) cconv_residual_norm_long_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  const T* resid = static_cast<const T*>(p.resid);
  const T* block = static_cast<const T*>(p.block);
  const T* gate = static_cast<const T*>(p.gate);
  const T* w_post = static_cast<const T*>(p.w_post);
  const T* w_pre = static_cast<const T*>(p.w_pre);
  T* resid_out = static_cast<T*>(p.resid_out);
  T* norm_out = static_cast<T*>(p.norm_out);
  const float inv_d = 1.0f / float(p.D);
  int buf = 0;
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    const T* r = resid + t * p.resid_rs;
    const T* y = block ? block + t * p.block_rs : nullptr;
    const T* g = gate ? gate + (p.rows_per_gate ? t / p.rows_per_gate : 0) * p.gate_rs : nullptr;
    float rho_y = 1.0f;
    if (y && w_post) {
      float ss = 0.0f;
      for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
        const float f = to_f32(y[c]);
        ss += f * f;
      }
      rho_y = rsqrtf(block_sum2(ss, 0.0f, smem, buf).x * inv_d + p.eps);
    }
    auto out = [&](int c) {
      float o = p.scale * to_f32(r[c]);
      if (y) {
        float n = to_f32(y[c]);
        if (w_post) n *= rho_y * to_f32(w_post[c]);
        if (g) n *= to_f32(g[c]);
        o += n;
      }
      return o;
    };
    float rho_r = 1.0f;
    if (norm_out) {
      float ss = 0.0f;
      for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
        const float o = out(c);
        ss += o * o;
      }
      rho_r = rsqrtf(block_sum2(ss, 0.0f, smem, buf).x * inv_d + p.eps);
    }
    for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
      const float o = out(c);
      resid_out[t * p.resid_out_rs + c] = from_f32<T>(o);
      if (norm_out) norm_out[t * p.norm_out_rs + c] = from_f32<T>(w_pre ? o * rho_r * to_f32(w_pre[c]) : o * rho_r);
    }
  }
}

// ---- backward ----------------------------------------------------------------------------------
// Block b takes the rows [T b / nb, T (b+1) / nb) in order and keeps its share of the column sums
// (dw_pre, dw_post, dgate of the current group) in registers.  At the end they go to its rows of the
// partial table part[b][4][D] (dw_pre, dw_post, gate group of its first row, gate group of its last
// row), which a second kernel adds up in a fixed order.  A gate group that lies inside one block's
// rows is complete there and written at once.
template <typename T>
__device__ __forceinline__ int64_t first_row(const NormParams& p, int64_t b) {
  return p.T * b / p.nb;
}

template <typename T, int E, int NV>
__global__ void __launch_bounds__(512) cconv_residual_norm_backward_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  using V = Vec<T, E>;
  const T* dres = static_cast<const T*>(p.dresid_out);  // may be dresid
  const T* __restrict__ dx = static_cast<const T*>(p.dnorm_out);
  const T* __restrict__ block = static_cast<const T*>(p.block);
  const T* __restrict__ resid_out = static_cast<const T*>(p.resid_out);
  const T* __restrict__ gate = static_cast<const T*>(p.gate);
  const T* __restrict__ w_post = static_cast<const T*>(p.w_post);
  const T* __restrict__ w_pre = static_cast<const T*>(p.w_pre);
  T* dresid = static_cast<T*>(p.dresid);
  T* dblock = static_cast<T*>(p.dblock);
  T* dgate = static_cast<T*>(p.dgate);
  const int nt = blockDim.x, tid = threadIdx.x;
  const float inv_d = 1.0f / float(p.D);
  const int64_t row0 = first_row<T>(p, blockIdx.x), row1 = first_row<T>(p, blockIdx.x + 1);
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T;
  float* part = p.part + int64_t(blockIdx.x) * 4 * p.D;
  int buf = 0;
  float s_pre[NV][E], s_post[NV][E], s_gate[NV][E];
  V vw_pre[NV], vw_post[NV], vgate[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * nt + tid) * E;
    vw_pre[v].zero();
    vw_post[v].zero();
    vgate[v].zero();
    if (c < p.D) {
      if (w_pre) vw_pre[v].load(w_pre + c);
      if (w_post) vw_post[v].load(w_post + c);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) s_pre[v][i] = s_post[v][i] = s_gate[v][i] = 0.0f;
  }
  int64_t group = row0 / per;
  const int64_t group0 = group;
  auto load_gate = [&]() {
    if (!gate) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      if (c < p.D) vgate[v].load(gate + group * p.gate_rs + c);
    }
  };
  // writes the sums of the group that ends (or that the block ends in), and starts the next
  auto flush_gate = [&]() {
    if (!gate) return;
    const int64_t g0 = group * per, g1 = g0 + per < p.T ? g0 + per : p.T;
    const bool whole = g0 >= row0 && g1 <= row1;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      if (c < p.D) {
        if (whole) {
          V::store(dgate + group * p.dgate_rs + c, s_gate[v]);
        } else {
          float* to = part + (group == group0 ? 2 : 3) * int64_t(p.D) + c;
#pragma unroll
          for (int i = 0; i < E; ++i) to[i] = s_gate[v][i];
        }
      }
#pragma unroll
      for (int i = 0; i < E; ++i) s_gate[v][i] = 0.0f;
    }
  };
  load_gate();
  V nr[NV], nd[NV], nx[NV], ny[NV];  // the row that is on its way
  auto fetch = [&](int64_t t) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      nr[v].zero();
      nd[v].zero();
      nx[v].zero();
      ny[v].zero();
      if (c < p.D) {
        if (dx) {
          nr[v].load(resid_out + t * p.resid_out_rs + c);
          nx[v].load(dx + t * p.dnorm_out_rs + c);
        }
        if (dres) nd[v].load(dres + t * p.dresid_out_rs + c);
        if (block) ny[v].load(block + t * p.block_rs + c);
      }
    }
  };
  if (row0 < row1) fetch(row0);
  for (int64_t t = row0; t < row1; ++t) {
    if (t / per != group) {
      flush_gate();
      group = t / per;
      load_gate();
    }
    V r[NV], x[NV], y[NV];
    float s[NV][E];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      r[v] = nr[v];
      x[v] = nx[v];
      y[v] = ny[v];
      nd[v].get(s[v]);
    }
    if (t + 1 < row1) fetch(t + 1);
    if (dx) {
      float srr = 0.0f, ser = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float fr[E], fx[E], fw[E];
        r[v].get(fr);
        x[v].get(fx);
        vw_pre[v].get(fw);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          srr += fr[i] * fr[i];
          ser += (w_pre ? fx[i] * fw[i] : fx[i]) * fr[i];
        }
      }
      const float2 q = block_sum2(srr, ser, smem, buf);
      const float rho = rsqrtf(q.x * inv_d + p.eps);
      const float k = rho * rho * rho * (q.y * inv_d);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float fr[E], fx[E], fw[E];
        r[v].get(fr);
        x[v].get(fx);
        vw_pre[v].get(fw);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          s[v][i] += rho * (w_pre ? fx[i] * fw[i] : fx[i]) - k * fr[i];
          s_pre[v][i] += fx[i] * (fr[i] * rho);
        }
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      float f[E];
#pragma unroll
      for (int i = 0; i < E; ++i) f[i] = p.scale * s[v][i];
      if (c < p.D) V::store(dresid + t * p.dresid_rs + c, f);
    }
    if (!block) continue;
    float rho = 1.0f, k = 0.0f;
    if (w_post) {
      float syy = 0.0f, sfy = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float fy[E], fg[E], fw[E];
        y[v].get(fy);
        vgate[v].get(fg);
        vw_post[v].get(fw);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          syy += fy[i] * fy[i];
          sfy += s[v][i] * (gate ? fg[i] : 1.0f) * fw[i] * fy[i];
        }
      }
      const float2 q = block_sum2(syy, sfy, smem, buf);
      rho = rsqrtf(q.x * inv_d + p.eps);
      k = rho * rho * rho * (q.y * inv_d);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      float fy[E], fg[E], fw[E], o[E];
      y[v].get(fy);
      vgate[v].get(fg);
      vw_post[v].get(fw);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float dn = gate ? fg[i] * s[v][i] : s[v][i];
        const float yhat = fy[i] * rho;
        if (gate) s_gate[v][i] += s[v][i] * (w_post ? yhat * fw[i] : yhat);
        s_post[v][i] += dn * yhat;
        o[i] = w_post ? rho * (dn * fw[i]) - k * fy[i] : dn;
      }
      if (c < p.D) V::store(dblock + t * p.dblock_rs + c, o);
    }
  }
  if (row0 < row1) flush_gate();
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * nt + tid) * E;
    if (c < p.D) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        part[c + i] = s_pre[v][i];
        part[p.D + c + i] = s_post[v][i];
      }
    }
  }
}

// Rows too long for registers: column sums live in the partial table (5 rows a block here; the fifth
// holds the sums of a gate group that is complete within the block until it is written).
template <typename T>
__global__ void __launch_bounds__(512) cconv_residual_norm_backward_long_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  const T* dres = static_cast<const T*>(p.dresid_out);
  const T* dx = static_cast<const T*>(p.dnorm_out);
  const T* block = static_cast<const T*>(p.block);
  const T* resid_out = static_cast<const T*>(p.resid_out);
  const T* gate = static_cast<const T*>(p.gate);
  const T* w_post = static_cast<const T*>(p.w_post);
  const T* w_pre = static_cast<const T*>(p.w_pre);
  T* dresid = static_cast<T*>(p.dresid);
  T* dblock = static_cast<T*>(p.dblock);
  T* dgate = static_cast<T*>(p.dgate);
  const float inv_d = 1.0f / float(p.D);
  const int64_t row0 = first_row<T>(p, blockIdx.x), row1 = first_row<T>(p, blockIdx.x + 1);
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T;
  float* part = p.part + int64_t(blockIdx.x) * 4 * p.D;
  float* whole_sum = p.part + (int64_t(p.nb) * 4 + blockIdx.x) * p.D;
  const int64_t group0 = row0 / per;
  int buf = 0;
  for (int c = threadIdx.x; c < p.D; c += blockDim.x) part[c] = part[p.D + c] = 0.0f;
  for (int64_t t = row0; t < row1; ++t) {
    const int64_t group = t / per;
    const int64_t g0 = group * per, g1 = g0 + per < p.T ? g0 + per : p.T;
    const bool whole = g0 >= row0 && g1 <= row1;
    float* gsum = whole ? whole_sum : part + (group == group0 ? 2 : 3) * int64_t(p.D);
    const bool starts = t == row0 || t == g0, ends = t + 1 == g1;
    const T* fr = resid_out + t * p.resid_out_rs;
    const T* fx = dx ? dx + t * p.dnorm_out_rs : nullptr;
    const T* fd = dres ? dres + t * p.dresid_out_rs : nullptr;
    const T* fy = block ? block + t * p.block_rs : nullptr;
    const T* fg = gate ? gate + group * p.gate_rs : nullptr;
    float rho = 1.0f, k = 0.0f;
    if (fx) {
      float srr = 0.0f, ser = 0.0f;
      for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
        const float r = to_f32(fr[c]);
        srr += r * r;
        ser += (w_pre ? to_f32(fx[c]) * to_f32(w_pre[c]) : to_f32(fx[c])) * r;
      }
      const float2 q = block_sum2(srr, ser, smem, buf);
      rho = rsqrtf(q.x * inv_d + p.eps);
      k = rho * rho * rho * (q.y * inv_d);
    }
    auto grad = [&](int c) {
      float s = fd ? to_f32(fd[c]) : 0.0f;
      if (fx) s += rho * (w_pre ? to_f32(fx[c]) * to_f32(w_pre[c]) : to_f32(fx[c])) - k * to_f32(fr[c]);
      return s;
    };
    float rho_y = 1.0f, ky = 0.0f;
    if (fy && w_post) {
      float syy = 0.0f, sfy = 0.0f;
      for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
        const float y = to_f32(fy[c]);
        syy += y * y;
        sfy += grad(c) * (fg ? to_f32(fg[c]) : 1.0f) * to_f32(w_post[c]) * y;
      }
      const float2 q = block_sum2(syy, sfy, smem, buf);
      rho_y = rsqrtf(q.x * inv_d + p.eps);
      ky = rho_y * rho_y * rho_y * (q.y * inv_d);
    }
    // a thread owns the columns c = threadIdx.x (mod blockDim.x) in every sweep, of all arrays
    for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
      const float s = grad(c);
      if (fx) part[c] += to_f32(fx[c]) * (to_f32(fr[c]) * rho);
      if (fy) {
        const float dn = fg ? to_f32(fg[c]) * s : s;
        const float yhat = to_f32(fy[c]) * rho_y;
        if (fg) {
          const float sum = (starts ? 0.0f : gsum[c]) + s * (w_post ? yhat * to_f32(w_post[c]) : yhat);
          gsum[c] = sum;
          if (whole && ends) dgate[group * p.dgate_rs + c] = from_f32<T>(sum);
        }
        part[p.D + c] += dn * yhat;
        dblock[t * p.dblock_rs + c] = from_f32<T>(w_post ? rho_y * (dn * to_f32(w_post[c])) - ky * to_f32(fy[c]) : dn);
      }
      dresid[t * p.dresid_rs + c] = from_f32<T>(p.scale * s);
    }
  }
}

// Adds up the partial table: blockIdx.y 0: dw_pre, 1: dw_post, 2 + i: a gate group that lies in
// several blocks -- group i, or where there are more groups than blocks the one that the rows of block
// i end in, if block i is the first that it lies in.  32 columns by 8 slices of the table a block.
template <typename T>
__global__ void __launch_bounds__(256) cconv_residual_norm_sums_kernel(const NormParams p) {
  __shared__ float smem[8][33];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T;
  int b0 = 0, b1 = p.nb - 1, slot = int(blockIdx.y);
  T* to = static_cast<T*>(blockIdx.y == 0 ? p.dw_pre : p.dw_post);
  int64_t group = 0;
  if (blockIdx.y >= 2) {
    // every block has a row (nb <= T); row t lies in block ceil((t + 1) nb / T) - 1
    const int i = int(blockIdx.y) - 2;
    group = p.sums_by_group ? i : (first_row<T>(p, i + 1) - 1) / per;
    const int64_t g0 = group * per, g1 = g0 + per < p.T ? g0 + per : p.T;
    b0 = int(((g0 + 1) * p.nb + p.T - 1) / p.T) - 1;
    b1 = int((g1 * p.nb + p.T - 1) / p.T) - 1;
    if (b0 == b1 || (!p.sums_by_group && b0 != i)) return;  // complete already; another block's
    to = static_cast<T*>(p.dgate) + group * p.dgate_rs;
  } else if (!to) {
    return;
  }
  float s = 0.0f;
  if (c < p.D) {
    for (int b = b0 + slice; b <= b1; b += 8) {
      int at = slot;
      if (blockIdx.y >= 2) at = first_row<T>(p, b) / per == group ? 2 : 3;
      s += p.part[(int64_t(b) * 4 + at) * p.D + c];
    }
  }
  smem[slice][threadIdx.x & 31] = s;
  __syncthreads();
  if (slice == 0 && c < p.D) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += smem[i][threadIdx.x];
    to[c] = from_f32<T>(s);
  }
}

// Threads a block and accesses a thread for rows of D elements taken E at a time: at most `held`
// elements a thread, whole warps, one access a thread as long as that leaves 256 threads or fewer.
struct Shape {
  int threads, nv;
};
Shape shape_of(int64_t D, int E, int held, int most) {
  const int64_t acc = cdiv64(D, E);
  int nv = 1;
  while (nv * E < held && acc > int64_t(nv) * 256) nv *= 2;
  const int64_t threads = round_up64(cdiv64(acc, nv), 32);
  return threads <= most ? Shape{int(threads), nv} : Shape{0, 0};
}

bool wide(const NormParams& p, int es, bool backward) {
  const int E = 16 / es;
  if (p.D % E) return false;
  uintptr_t all = 0;
  int64_t strides = 0;
  auto add = [&](const void* q, int64_t rs) {
    if (!q) return;
    all |= reinterpret_cast<uintptr_t>(q);
    strides |= rs * es;
  };
  add(p.block, p.block_rs);
  add(p.gate, p.gate_rs);
  add(p.w_post, 0);
  add(p.w_pre, 0);
  add(p.resid_out, p.resid_out_rs);
  if (backward) {
    add(p.dresid_out, p.dresid_out_rs);
    add(p.dnorm_out, p.dnorm_out_rs);
    add(p.dresid, p.dresid_rs);
    add(p.dblock, p.dblock_rs);
    add(p.dgate, p.dgate_rs);
  } else {
    add(p.resid, p.resid_rs);
    add(p.norm_out, p.norm_out_rs);
  }
  return ((all | uintptr_t(strides)) & 15u) == 0;
}

template <typename T, int E, int NV>
void launch_forward_nv(const NormParams& p, int threads, int64_t grid, cudaStream_t s) {
  cconv_residual_norm_kernel<T, E, NV><<<unsigned(grid), threads, 0, s>>>(p);
}

template <typename T>
cudaError_t launch_forward(const NormParams& p, int sms, cudaStream_t s) {
  constexpr int kWide = 16 / int(sizeof(T));
  const bool w = wide(p, sizeof(T), false);
  const Shape sh = shape_of(p.D, w ? kWide : 1, 16, 1024);
  const int threads = sh.threads ? sh.threads : 1024;
  const int64_t grid = std::min<int64_t>(p.T, int64_t(sms) * std::max(1, std::min(32, 1024 / threads)));
  if (!sh.threads) {
    cconv_residual_norm_long_kernel<T><<<unsigned(grid), threads, 0, s>>>(p);
  } else if (w) {
    if (sh.nv == 1) launch_forward_nv<T, kWide, 1>(p, threads, grid, s);
    else if (sh.nv == 2) launch_forward_nv<T, kWide, 2>(p, threads, grid, s);
    else launch_forward_nv<T, kWide, sizeof(T) == 4 ? 4 : 2>(p, threads, grid, s);
  } else {
    if (sh.nv == 1) launch_forward_nv<T, 1, 1>(p, threads, grid, s);
    else if (sh.nv == 2) launch_forward_nv<T, 1, 2>(p, threads, grid, s);
    else if (sh.nv == 4) launch_forward_nv<T, 1, 4>(p, threads, grid, s);
    else if (sh.nv == 8) launch_forward_nv<T, 1, 8>(p, threads, grid, s);
    else launch_forward_nv<T, 1, 16>(p, threads, grid, s);
  }
  return cudaGetLastError();
}

template <typename T, int E, int NV>
void launch_backward_nv(const NormParams& p, int threads, cudaStream_t s) {
  cconv_residual_norm_backward_kernel<T, E, NV><<<unsigned(p.nb), threads, 0, s>>>(p);
}

template <typename T>
cudaError_t launch_backward(const NormParams& p, cudaStream_t s) {
  constexpr int kWide = 16 / int(sizeof(T));
  const bool w = wide(p, sizeof(T), true);
  const Shape sh = shape_of(p.D, w ? kWide : 1, 16, 512);
  if (!sh.threads) {
    cconv_residual_norm_backward_long_kernel<T><<<unsigned(p.nb), 512, 0, s>>>(p);
  } else if (w) {
    if (sh.nv == 1) launch_backward_nv<T, kWide, 1>(p, sh.threads, s);
    else if (sh.nv == 2) launch_backward_nv<T, kWide, 2>(p, sh.threads, s);
    else launch_backward_nv<T, kWide, sizeof(T) == 4 ? 4 : 2>(p, sh.threads, s);
  } else {
    if (sh.nv == 1) launch_backward_nv<T, 1, 1>(p, sh.threads, s);
    else if (sh.nv == 2) launch_backward_nv<T, 1, 2>(p, sh.threads, s);
    else if (sh.nv == 4) launch_backward_nv<T, 1, 4>(p, sh.threads, s);
    else if (sh.nv == 8) launch_backward_nv<T, 1, 8>(p, sh.threads, s);
    else launch_backward_nv<T, 1, 16>(p, sh.threads, s);
  }
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  NormParams q = p;
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T, groups = cdiv64(p.T, per);
  q.sums_by_group = groups <= p.nb;
  const int64_t items = !p.gate || per == 1 ? 0 : q.sums_by_group ? groups : p.nb - 1;
  const dim3 grid(unsigned(cdiv64(p.D, 32)), unsigned(2 + items));
  cconv_residual_norm_sums_kernel<T><<<grid, 256, 0, s>>>(q);
  return cudaGetLastError();
}

}  // namespace

int norm_backward_blocks(int64_t T, int64_t D, int sms) {
  // about 512 threads of rows an SM: rows in flight cover the latency of HBM, and the table of
  // partial sums stays small against the arrays
  const int64_t threads = std::max<int64_t>(32, std::min<int64_t>(512, round_up64(cdiv64(D, 16), 32)));
  return int(std::max<int64_t>(1, std::min<int64_t>(T, int64_t(sms) * std::min<int64_t>(16, 512 / threads))));
}

cudaError_t run_norm_forward(const NormParams& p, int dtype, int sms, cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16) return launch_forward<__nv_bfloat16>(p, sms, s);
  if (dtype == CCONV_TYPE_FP16) return launch_forward<__half>(p, sms, s);
  return launch_forward<float>(p, sms, s);
}

cudaError_t run_norm_backward(const NormParams& p, int dtype, cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16) return launch_backward<__nv_bfloat16>(p, s);
  if (dtype == CCONV_TYPE_FP16) return launch_backward<__half>(p, s);
  return launch_backward<float>(p, s);
}

}  // namespace cconv
