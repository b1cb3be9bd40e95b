// Norms before and after a block, fused with the block's gate and the residual scale.
//
//   forward    n = y rho_y w_post,  r' = scale r + gate n,  x = r' rho_r w_pre,
//              rho_v = 1 / sqrt(mean(v^2) + eps)
//   backward   e = dx w_pre,  S = dr' + rho_r e - r' rho_r^3 mean(e r')       (dL/dr', all of it)
//              dr = scale S,  dgate = sum_t S n,  dn = gate S
//              f = dn w_post,  dy = rho_y f - y rho_y^3 mean(f y)
//              dw_post = sum_t dn y rho_y,  dw_pre = sum_t dx r' rho_r
//   (rho^3 mean is formed from the mean on, a rho at a time: rho^3 alone leaves fp32's range for rows of 1e13 or an eps of 1e-26)
//
// Both directions read every [T][D] array once from memory and write every output once; a row stays on chip, in
// registers or in shared memory, between its two reductions (over y, then over r'; backward: over r' and e, then
// over y and f), so they are bound by HBM.  That holds forward up to 16384 channels, and backward up to 65536 where a
// block or a cluster of them has room for the row; the *_long_ kernels, for the rest, read a row once for
// each sweep over it.  Measured, 16384 x 4096 bf16 with 8 gates: forward 89.5 us, 6.0 TB/s (4 arrays once: 82 us
// at the rate of a copy); backward 147 us, 5.5 TB/s (6 arrays: 123 us), 135 of them the first kernel.  One token
// of 4096 channels: 2.5 us on the device.
#include <algorithm>
#include <type_traits>

#include "block.h"
#include "block_device.cuh"
#include "block_launch.h"
#include "block_norm.h"
#include "host_setup.h"
#include "ptx_sm100.cuh"

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

// Block b of the kernels that take neighbouring rows has the rows [T b / nb, T (b+1) / nb).
__device__ __forceinline__ int64_t first_row(const NormParams& p, int64_t b) {
  return p.T * b / p.nb;
}

// A ring in shared memory for rows that begin anywhere: a bulk copy brings the 16-byte pieces that a row lies
// in, so that its first element lies as far behind the slot's start as in memory behind a multiple of 16.  Pieces
// that reach out of the whole array (of its first and last row) stay behind; complete() fetches their elements.
template <typename T, int kArrays>
struct RowRing {
  struct Span {
    uintptr_t row, end, lo, hi;  // of the row; of the pieces that are copied
  };
  const T* base[kArrays];  // null: absent
  int64_t rs[kArrays];
  int64_t rows_of_all, row0, row1;
  uint32_t row_bytes, slot, ring0, full0, stages;

  __device__ __forceinline__ Span span(int a, int64_t t) const {
    Span s;
    const uintptr_t first = reinterpret_cast<uintptr_t>(base[a]);
    s.row = first + uintptr_t(t * rs[a]) * sizeof(T);
    s.end = s.row + row_bytes;
    s.lo = s.row & ~uintptr_t(15);
    s.hi = (s.end + 15) & ~uintptr_t(15);
    if (s.lo < first) s.lo += 16;
    if (s.hi > first + uintptr_t((rows_of_all - 1) * rs[a]) * sizeof(T) + row_bytes) s.hi -= 16;
    return s;
  }
  __device__ __forceinline__ void copy(int64_t t) const {  // one thread
    const uint32_t st = uint32_t(t - row0) % stages, bar = full0 + 8 * st, to = ring0 + st * kArrays * slot;
    uint32_t bytes = 0;
#pragma unroll
    for (int a = 0; a < kArrays; ++a) {
      if (!base[a]) continue;
      const Span s = span(a, t);
      bytes += uint32_t(s.hi - s.lo);
    }
    mbar_arrive_expect_tx(bar, bytes);
#pragma unroll
    for (int a = 0; a < kArrays; ++a) {
      if (!base[a]) continue;
      const Span s = span(a, t);
      bulk_load(to + a * slot + uint32_t(s.lo - (s.row & ~uintptr_t(15))), reinterpret_cast<const void*>(s.lo),
                uint32_t(s.hi - s.lo), bar);
    }
  }
  __device__ __forceinline__ void begin() const {  // one thread
    for (uint32_t i = 0; i < stages; ++i) mbar_init(full0 + 8 * i, 1);
    fence_barrier_init();
    for (int64_t t = row0; t < row1 && t < row0 + int64_t(stages); ++t) copy(t);
  }
  // Array a of row t, which lies in stage st.
  __device__ __forceinline__ T* row(uint8_t* ring, int a, uint32_t st, int64_t t) const {
    const uintptr_t at = reinterpret_cast<uintptr_t>(base[a] + t * rs[a]);
    return reinterpret_cast<T*>(ring + (st * kArrays + a) * slot + (at & 15));
  }
  // All threads, once the copies of row t have landed.
  __device__ __forceinline__ void complete(uint8_t* ring, uint32_t st, int64_t t) const {
    if (t != 0 && t != rows_of_all - 1) return;
#pragma unroll
    for (int a = 0; a < kArrays; ++a) {
      if (!base[a]) continue;
      const Span s = span(a, t);
      const uint32_t n = row_bytes / sizeof(T), head = s.lo > s.row ? uint32_t(s.lo - s.row) / sizeof(T) : 0,
                     tail = s.end > s.hi ? uint32_t(s.end - s.hi) / sizeof(T) : 0;
      if (threadIdx.x < head) row(ring, a, st, t)[threadIdx.x] = base[a][t * rs[a] + threadIdx.x];
      if (threadIdx.x < tail) row(ring, a, st, t)[n - 1 - threadIdx.x] = base[a][t * rs[a] + n - 1 - threadIdx.x];
    }
    fence_proxy_async_smem();  // the next copy into the slot comes after
    __syncthreads();
  }
};

// Rows of which a thread takes the elements v nt + tid.  kThreads: the threads of a block, if known when compiled;
// a row then has more than kThreads NV 2/3 elements (NV = 12 and 16), so that most need no comparison.
template <int NV, int kThreads>
struct Across {
  static constexpr int kSure = kThreads && NV > 8 ? NV - 4 : 0;  // elements that every thread has
  static __device__ __forceinline__ int nt() { return kThreads ? kThreads : blockDim.x; }
  static __device__ __forceinline__ int column(int v) { return v * nt() + int(threadIdx.x); }
  static __device__ __forceinline__ bool inside(int v, int D) { return v < kSure || column(v) < D; }
};
// Elements of a row (`otherwise` where it ends, or where there is none): loads without conditions, so that all are on
// their way together.  kSpare: memory goes on behind the row.
template <int kThreads, bool kSpare, typename T, int NV>
__device__ __forceinline__ void load_across(float (&f)[NV], const T* from, int D, float otherwise) {
  using A = Across<NV, kThreads>;
  if (from) {
    T raw[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = from[kSpare || v < A::kSure ? A::column(v) : min(A::column(v), D - 1)];
#pragma unroll
    for (int v = 0; v < NV; ++v) f[v] = A::inside(v, D) ? to_f32(raw[v]) : otherwise;
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) f[v] = otherwise;
  }
}

// ---- forward -----------------------------------------------------------------------------------
// A block a row (and the row gridDim.x further on, ...): few rows, whose latency counts, or rows that are not
// wide.  Everything that a row needs is asked for before its first reduction (one row of 4096: 2.5 us).
template <typename T, int E, int NV>
__global__ void __launch_bounds__(1024) cconv_residual_norm_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  start_in_order();
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
  V vpost[NV], vpre[NV];
  auto fetch = [&](V& v, const T* from, int c) {
    v.zero();
    if (from && c < p.D) v.load(from + c);
  };
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    fetch(vpost[v], w_post, (v * nt + tid) * E);
    fetch(vpre[v], w_pre, (v * nt + tid) * E);
  }
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    const T* row_r = resid + t * p.resid_rs;
    const T* row_y = block ? block + t * p.block_rs : nullptr;
    const T* row_g = gate ? gate + (p.rows_per_gate ? t / p.rows_per_gate : 0) * p.gate_rs : nullptr;
    V r[NV], y[NV], g[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      fetch(r[v], row_r, c);
      fetch(y[v], row_y, c);
      fetch(g[v], row_g, c);
    }
    float rho = 1.0f;
    if (block && w_post) {
      float ss = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float f[E];
        y[v].get(f);
#pragma unroll
        for (int i = 0; i < E; ++i) ss += f[i] * f[i];
      }
      rho = rsqrtf(block_sum2(ss, 0.0f, smem, buf).x * inv_d + p.eps);
    }
    float o[NV][E], ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      float f[E];
      r[v].get(o[v]);
      y[v].get(f);
      if (w_post) {
        float w[E];
        vpost[v].get(w);
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] *= rho * w[i];
      }
      if (gate) {
        float w[E];
        g[v].get(w);
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] *= w[i];
      }
#pragma unroll
      for (int i = 0; i < E; ++i) {
        o[v][i] = p.scale * o[v][i] + f[i];
        ss += o[v][i] * o[v][i];
      }
      if (c < p.D) V::store(resid_out + t * p.resid_out_rs + c, o[v]);
    }
    if (!norm_out) continue;
    rho = rsqrtf(block_sum2(ss, 0.0f, smem, buf).x * inv_d + p.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      float w[E];
      vpre[v].get(w);
#pragma unroll
      for (int i = 0; i < E; ++i) o[v][i] *= w_pre ? rho * w[i] : rho;
      if (c < p.D) V::store(norm_out + t * p.norm_out_rs + c, o[v]);
    }
  }
}

// Rows too long for registers: the row is read again in each of the three sweeps (from L2, which sets the pace:
// nothing of a row is kept on chip but its sums, so that any length works).
template <typename T>
__global__ void __launch_bounds__(1024) cconv_residual_norm_long_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  start_in_order();
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

// Many rows that are not wide, through the ring above (16384 x 4095 bf16: 131 us, 224 with a block size known at
// the launch; with a block a row and everything from global memory 516 us).
template <typename T, int NV, int kThreads>
__global__ void __launch_bounds__(kThreads) cconv_residual_norm_narrow_kernel(const NormParams p) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ float2 smem[2][32];
  __shared__ __align__(8) uint64_t full[8];
  __shared__ int abort_flag;
  start_in_order();
  const T* block = static_cast<const T*>(p.block);
  const T* __restrict__ gate = static_cast<const T*>(p.gate);
  const T* __restrict__ w_post = static_cast<const T*>(p.w_post);
  const T* __restrict__ w_pre = static_cast<const T*>(p.w_pre);
  T* resid_out = static_cast<T*>(p.resid_out);
  T* norm_out = static_cast<T*>(p.norm_out);
  using A = Across<NV, kThreads>;
  const int tid = threadIdx.x;
  const float inv_d = 1.0f / float(p.D);
  const int64_t row0 = first_row(p, blockIdx.x), row1 = first_row(p, blockIdx.x + 1);
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T;
  const RowRing<T, 2> rows = {{static_cast<const T*>(p.resid), block}, {p.resid_rs, p.block_rs}, p.T, row0, row1,
                              uint32_t(p.D * sizeof(T)), p.ring_slot, smem_u32(ring), smem_u32(full), uint32_t(p.ring_rows)};
  if (tid == 0) {
    abort_flag = 0;
    rows.begin();
  }
  __syncthreads();
  float gw[NV], wpre[NV];  // gate * w_post of the current group; w_pre
  load_across<kThreads, false>(wpre, w_pre, p.D, 1.0f);
  int64_t group_end = row0;
  uint32_t st = 0, phase = 0;
  int buf = 0;
  int64_t t = row0;
  for (; t < row1; ++t) {
    if (t == group_end || t == row0) {
      const int64_t group = t / per;
      group_end = (group + 1) * per;
      float g[NV];
      load_across<kThreads, false>(g, gate ? gate + group * p.gate_rs : nullptr, p.D, 1.0f);
      load_across<kThreads, false>(gw, w_post, p.D, 1.0f);
#pragma unroll
      for (int v = 0; v < NV; ++v) gw[v] *= g[v];
    }
    const bool ok = mbar_wait(rows.full0 + 8 * st, phase, &abort_flag, p.status, kStatProducerWait, p.limit_ns);
    // every thread is past the row before: its place in the ring is free
    if (!__syncthreads_and(ok)) break;
    if (tid == 0 && t > row0 && t - 1 + p.ring_rows < row1) rows.copy(t - 1 + p.ring_rows);
    rows.complete(ring, st, t);
    const T* row_r = rows.row(ring, 0, st, t);
    const T* row_y = block ? rows.row(ring, 1, st, t) : nullptr;
    if (++st == uint32_t(p.ring_rows)) st = 0, phase ^= 1;
    float rho = 1.0f, ss = 0.0f;
    float o[NV];
    load_across<kThreads, true>(o, row_y, p.D, 0.0f);
    if (block && w_post) {
#pragma unroll
      for (int v = 0; v < NV; ++v) ss += o[v] * o[v];
      rho = rsqrtf(block_sum2(ss, 0.0f, smem, buf).x * inv_d + p.eps);
      ss = 0.0f;
    }
    float r[NV];
    load_across<kThreads, true>(r, row_r, p.D, 0.0f);
    T* to = resid_out + t * p.resid_out_rs;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      o[v] = p.scale * r[v] + o[v] * (rho * gw[v]);
      ss += o[v] * o[v];
      if (A::inside(v, p.D)) to[A::column(v)] = from_f32<T>(o[v]);
    }
    if (!norm_out) continue;
    rho = rsqrtf(block_sum2(ss, 0.0f, smem, buf).x * inv_d + p.eps);
    to = norm_out + t * p.norm_out_rs;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (A::inside(v, p.D)) to[A::column(v)] = from_f32<T>(o[v] * (rho * wpre[v]));
  }
  if (t < row1) {  // a copy did not come in time: let those on their way land
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000) {
    }
  }
}

// ---- backward ----------------------------------------------------------------------------------
// A block takes its rows in order and keeps its share of the column sums
// (dw_pre, dw_post, dgate of the current group) in registers.  At the end they go to its rows of the
// partial table part[b][4][D] (dw_pre, dw_post, gate group of its first row, gate group of its last
// row), which a second kernel adds up in a fixed order.  A gate group that lies inside one block's
// rows is complete there and written at once.
// Rows that are not wide (an odd length, pitch or address): element v nt + tid is the thread's, so that the
// narrow accesses of a warp are neighbours.  kThreads: rows come through the ring above, and a block's size is
// known when compiled, which leaves accesses no address arithmetic of their own (16384 x 4095 bf16: 259 us, and 490
// with a size known at the launch); 0: straight from global memory, where rows are few or the ring has no room for
// two (1118 us).  kCluster: rows too long for one block's registers are shared by the 2, 4 or 8 blocks of a
// cluster, a range of columns each, which exchange their sums through distributed shared memory (4096 x 16384
// bf16: 345 us; with sums in memory, cconv_residual_norm_backward_long_kernel, 2860 us).
constexpr int kMostParts = 8;
template <typename T, int NV, int kThreads, bool kCluster = false>
__global__ void __launch_bounds__(kThreads ? kThreads : 512, 512 / (kThreads ? kThreads : 512)) cconv_residual_norm_backward_kernel(const NormParams p) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ float2 smem[2][32];
  __shared__ __align__(8) uint64_t full[8];
  __shared__ int abort_flag;
  __shared__ float2 shares[2][kMostParts];
  start_in_order();
  using A = Across<NV, kThreads>;
  constexpr bool kRing = kThreads != 0;
  const int parts = kCluster ? p.parts : 1, rank = kCluster ? int(cluster_ctarank()) : 0;
  const int b = kCluster ? int(blockIdx.x) / parts : int(blockIdx.x);
  const int c0 = kCluster ? int(int64_t(p.D) * rank / parts) : 0;
  const int D = kCluster ? int(int64_t(p.D) * (rank + 1) / parts) - c0 : p.D;  // the block's columns, from c0 on
  auto columns = [&](const void* q) { return static_cast<const T*>(q) + (kCluster && q ? c0 : 0); };
  const T* dres = columns(p.dresid_out);  // may be dresid
  const T* __restrict__ dx = columns(p.dnorm_out);
  const T* __restrict__ block = columns(p.block);
  const T* __restrict__ resid_out = columns(p.resid_out);
  const T* __restrict__ gate = columns(p.gate);
  const T* __restrict__ w_post = columns(p.w_post);
  const T* __restrict__ w_pre = columns(p.w_pre);
  T* dresid = static_cast<T*>(p.dresid) + c0;
  T* dblock = static_cast<T*>(p.dblock) + c0;
  T* dgate = static_cast<T*>(p.dgate) + c0;
  const int tid = threadIdx.x;
  const float inv_d = 1.0f / float(p.D);
  const int64_t row0 = first_row(p, b), row1 = first_row(p, b + 1);
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T;
  float* part = p.part + int64_t(b) * 4 * p.D + c0;
  int buf = 0, shares_of = 0;
  // Sums over the whole row: of the block, and then, in the order of the ranks, of the cluster.
  auto row_sum2 = [&](float f, float g) {
    float2 q = block_sum2(f, g, smem, buf);
    if (kCluster) {
      if (tid < parts) st_cluster_v2(cluster_map_shared(smem_u32(&shares[shares_of][rank]), tid), q.x, q.y);
      __syncwarp();
      cluster_sync_all();
      q = shares[shares_of][0];
      for (int i = 1; i < parts; ++i) q.x += shares[shares_of][i].x, q.y += shares[shares_of][i].y;
      shares_of ^= 1;
    }
    return q;
  };
  // Sums over rows: x rhat; S yhat of the current gate group (dgate is w_post of it); dw_post (gate times
  // each group's S yhat, added when the group ends).
  // Those of dw_post, which change only where a group ends, lie in the partial table (each thread touches its own
  // columns alone).
  float s_pre[NV], s_group[NV], gw[NV];  // gw: gate * w_post of the current group
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    s_pre[v] = s_group[v] = gw[v] = 0.0f;
    if (A::inside(v, D)) part[p.D + A::column(v)] = 0.0f;
  }
  int64_t group = row0 / per, group_end = (group + 1) * per;
  const int64_t group0 = group;
  auto start_group = [&]() {
    float g[NV];
    load_across<kThreads, false>(g, gate ? gate + group * p.gate_rs : nullptr, D, 1.0f);
    load_across<kThreads, false>(gw, w_post, D, 1.0f);
#pragma unroll
    for (int v = 0; v < NV; ++v) gw[v] *= g[v];
  };
  // adds the group that ends (or that the block ends in) to dw_post and writes its part of dgate
  auto end_group = [&]() {
    const int64_t g0 = group * per, g1 = group_end < p.T ? group_end : p.T;
    const bool whole = g0 >= row0 && g1 <= row1;
    float g[NV], w[NV];
    load_across<kThreads, false>(g, gate ? gate + group * p.gate_rs : nullptr, D, 1.0f);
    load_across<kThreads, false>(w, w_post, D, 1.0f);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = A::column(v);
      if (A::inside(v, D)) part[p.D + c] += g[v] * s_group[v];
      const float f = w[v] * s_group[v];
      s_group[v] = 0.0f;
      if (gate && A::inside(v, D)) {
        if (whole) dgate[group * p.dgate_rs + c] = from_f32<T>(f);
        else part[(group == group0 ? 2 : 3) * int64_t(p.D) + c] = f;
      }
    }
  };
  RowRing<T, 4> rows;  // r', dx, dr', y
  const T* pre = w_pre;
  if (kRing) {
    rows = {{dx ? resid_out : nullptr, dx, dres, block},
            {p.resid_out_rs, p.dnorm_out_rs, p.dresid_out_rs, p.block_rs},
            p.T, row0, row1, uint32_t(D * sizeof(T)), p.ring_slot, smem_u32(ring), smem_u32(full), uint32_t(p.ring_rows)};
    if (tid == 0) {
      abort_flag = 0;
      rows.begin();
    }
    if (w_pre) {  // a copy behind the ring
      T* w = reinterpret_cast<T*>(ring + p.ring_rows * 4 * p.ring_slot);
      for (int c = tid; c < D; c += kThreads) w[c] = w_pre[c];
      pre = w;
    }
    __syncthreads();
    if (kCluster) cluster_sync_all();  // the others' shared memory is there
  }
  start_group();
  uint32_t st = 0, phase = 0;
  bool dead = false;  // a copy did not come in time: a cluster's blocks go on, for the others wait for them
  int64_t t = row0;
  for (; t < row1; ++t) {
    const T* row_d = dres ? dres + t * p.dresid_out_rs : nullptr;
    const T* row_y = block ? block + t * p.block_rs : nullptr;
    const T* row_r = dx ? resid_out + t * p.resid_out_rs : nullptr;
    const T* row_x = dx ? dx + t * p.dnorm_out_rs : nullptr;
    if (kRing) {
      const bool ok = (kCluster && dead) || mbar_wait(rows.full0 + 8 * st, phase, &abort_flag, p.status, kStatProducerWait, p.limit_ns);
      // every thread is past the row before: its place in the ring is free
      if (!__syncthreads_and(ok)) {
        if (!kCluster) break;
        dead = true;
      }
      if (tid == 0 && !(kCluster && dead) && t > row0 && t - 1 + p.ring_rows < row1) rows.copy(t - 1 + p.ring_rows);
      rows.complete(ring, st, t);
      if (dx) row_r = rows.row(ring, 0, st, t), row_x = rows.row(ring, 1, st, t);
      if (dres) row_d = rows.row(ring, 2, st, t);
      if (block) row_y = rows.row(ring, 3, st, t);
      if (++st == uint32_t(p.ring_rows)) st = 0, phase ^= 1;
    }
    if (t == group_end) {
      end_group();
      ++group;
      group_end += per;
      start_group();
    }
    float s[NV];
    if (dx) {
      float r[NV], x[NV], w[NV], srr = 0.0f, ser = 0.0f;
      load_across<kThreads, kRing>(r, row_r, D, 0.0f);
      load_across<kThreads, kRing>(x, row_x, D, 0.0f);
      load_across<kThreads, kRing>(w, pre, D, 1.0f);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        srr += r[v] * r[v];
        ser += x[v] * w[v] * r[v];
      }
      const float2 q = row_sum2(srr, ser);
      const float rho = rsqrtf(q.x * inv_d + p.eps);
      const float k = rho * (rho * (rho * (q.y * inv_d)));
      // (read again: the reduction would hold them in registers that the sums need)
      load_across<kThreads, kRing>(r, row_r, D, 0.0f);
      load_across<kThreads, kRing>(x, row_x, D, 0.0f);
      load_across<kThreads, kRing>(w, pre, D, 1.0f);
      load_across<kThreads, kRing>(s, row_d, D, 0.0f);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        s[v] += rho * (x[v] * w[v]) - k * r[v];
        s_pre[v] += x[v] * (r[v] * rho);
      }
    } else {
      load_across<kThreads, kRing>(s, row_d, D, 0.0f);
    }
    T* const to_r = dresid + t * p.dresid_rs;
    float y[NV], syy = 0.0f, sfy = 0.0f;
    load_across<kThreads, kRing>(y, row_y, D, 0.0f);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = A::column(v);
      syy += y[v] * y[v];
      sfy += s[v] * gw[v] * y[v];
      if (A::inside(v, D)) to_r[c] = from_f32<T>(p.scale * s[v]);
    }
    if (!block) continue;
    T* const to_y = dblock + t * p.dblock_rs;
    float rho = 1.0f, k = 0.0f;
    if (w_post) {
      const float2 q = row_sum2(syy, sfy);
      rho = rsqrtf(q.x * inv_d + p.eps);
      k = rho * (rho * (rho * (q.y * inv_d)));
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = A::column(v);
      const float f = s[v] * gw[v];
      s_group[v] += s[v] * (y[v] * rho);
      if (A::inside(v, D)) to_y[c] = from_f32<T>(w_post ? rho * f - k * y[v] : f);  // (y may be infinite)
    }
  }
  if (t < row1 || dead) {  // let the copies that are on their way land
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000) {
    }
    return;
  }
  if (row0 < row1) end_group();
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = A::column(v);
    if (A::inside(v, D)) part[c] = s_pre[v];
  }
}

__device__ __forceinline__ float sum_of(uint64_t v) {
  const float2 f = halves_of(v);
  return f.x + f.y;
}
// 16 bytes of elements as pairs, and back.
template <typename T>
__device__ __forceinline__ void get_pairs(const void* from, uint64_t (&f)[16 / sizeof(T) / 2]) {
  const uint4 w = *static_cast<const uint4*>(from);
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
  if constexpr (sizeof(T) == 4) {
    f[0] = pair_of(__uint_as_float(a[0]), __uint_as_float(a[1]));
    f[1] = pair_of(__uint_as_float(a[2]), __uint_as_float(a[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = unpack2<T>(a[i]);
      f[i] = pair_of(v.x, v.y);
    }
  }
}
template <typename T>
__device__ __forceinline__ void put_pairs(void* to, const uint64_t (&f)[16 / sizeof(T) / 2]) {
  uint32_t a[4];
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 v = halves_of(f[i]);
      a[2 * i] = __float_as_uint(v.x);
      a[2 * i + 1] = __float_as_uint(v.y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = halves_of(f[i]);
      a[i] = pack2<T>(v.x, v.y);
    }
  }
  *static_cast<uint4*>(to) = make_uint4(a[0], a[1], a[2], a[3]);
}

// Wide rows: a ring in shared memory that bulk copies fill several rows ahead, so that no registers are
// held for what is on its way; 16 bytes of a row a thread and access, NV of them.  The arithmetic runs on
// pairs (8.5 operations an element instead of 17: with single ones issue slots, not HBM, set the pace).
// kAll: every array is given and the accesses cover the row exactly, as in a training step.  kPost: the block is
// normed (without, its gradient may not touch its values, which may be infinite; chosen at run time instead, 8192 x
// 6000 bf16 takes 169 us, not 164).
template <typename T, int NV, bool kAll, bool kPost>
__global__ void __launch_bounds__(512) cconv_residual_norm_backward_ring_kernel(const NormParams p) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ float2 smem[2][32];
  __shared__ __align__(8) uint64_t full[8];
  __shared__ int abort_flag;
  start_in_order();
  constexpr int E = 16 / int(sizeof(T)), P = E / 2;
  const T* dres = static_cast<const T*>(p.dresid_out);  // may be dresid
  const T* dx = static_cast<const T*>(p.dnorm_out);
  const T* block = static_cast<const T*>(p.block);
  const T* resid_out = static_cast<const T*>(p.resid_out);
  const T* __restrict__ gate = static_cast<const T*>(p.gate);
  const T* __restrict__ w_post = static_cast<const T*>(p.w_post);
  const T* __restrict__ w_pre = static_cast<const T*>(p.w_pre);
  T* dresid = static_cast<T*>(p.dresid);
  T* dblock = static_cast<T*>(p.dblock);
  T* dgate = static_cast<T*>(p.dgate);
  const int nt = blockDim.x, tid = threadIdx.x;
  const bool has_dx = kAll || dx, has_dres = kAll || dres, has_block = kAll || block;
  const bool has_pre = kAll || w_pre, has_gate = kAll || gate;
  auto inside = [&](int v) { return kAll || (v * nt + tid) * E < p.D; };
  const float inv_d = 1.0f / float(p.D);
  const int64_t row0 = first_row(p, blockIdx.x), row1 = first_row(p, blockIdx.x + 1);
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T;
  float* part = p.part + int64_t(blockIdx.x) * 4 * p.D;
  const uint32_t row_bytes = uint32_t(p.D) * sizeof(T), ring0 = smem_u32(ring), full0 = smem_u32(full);
  const uint64_t one = pair_of(1.0f, 1.0f), scale = pair_of(p.scale, p.scale);
  int buf = 0;
  // Sums over rows, as in the kernel above.  Those of dw_post, which change only where a group ends, lie
  // behind the ring (each thread touches its own columns alone).
  uint64_t s_pre[NV][P], s_group[NV][P], gw[NV][P];
  float* s_post = reinterpret_cast<float*>(ring + p.ring_rows * 4 * row_bytes);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int i = 0; i < P; ++i) s_pre[v][i] = s_group[v][i] = gw[v][i] = 0;
    if (inside(v)) {
#pragma unroll
      for (int i = 0; i < E; ++i) s_post[(v * nt + tid) * E + i] = 0.0f;
    }
  }
  int64_t group = row0 / per, group_end = (group + 1) * per;
  const int64_t group0 = group;
  auto get = [&](bool given, const T* from, int v, uint64_t (&f)[P], uint64_t otherwise) {
    if (given && inside(v)) {
      get_pairs<T>(from + (v * nt + tid) * E, f);
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) f[i] = otherwise;
    }
  };
  auto start_group = [&]() {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      uint64_t fg[P], fw[P];
      get(has_gate, gate + group * p.gate_rs, v, fg, one);
      get(kPost, w_post, v, fw, one);
#pragma unroll
      for (int i = 0; i < P; ++i) gw[v][i] = mul2(fg[i], fw[i]);
    }
  };
  auto end_group = [&]() {
    const int64_t g0 = group * per, g1 = group_end < p.T ? group_end : p.T;
    const bool whole = g0 >= row0 && g1 <= row1;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      uint64_t fg[P], fw[P];
      get(has_gate, gate + group * p.gate_rs, v, fg, one);
      get(kPost, w_post, v, fw, one);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (inside(v)) {
          const float2 q = halves_of(mul2(fg[i], s_group[v][i]));
          s_post[c + 2 * i] += q.x;
          s_post[c + 2 * i + 1] += q.y;
        }
        fw[i] = mul2(fw[i], s_group[v][i]);
        s_group[v][i] = 0;
      }
      if (has_gate && inside(v)) {
        if (whole) {
          put_pairs<T>(dgate + group * p.dgate_rs + c, fw);
        } else {
          float* to = part + (group == group0 ? 2 : 3) * int64_t(p.D) + c;
#pragma unroll
          for (int i = 0; i < P; ++i) *reinterpret_cast<uint64_t*>(to + 2 * i) = fw[i];
        }
      }
    }
  };
  // arrays of a row in the ring: r', dx, dr', y (those that are given)
  auto copy_row = [&](int64_t t) {
    const uint32_t st = uint32_t(t - row0) % uint32_t(p.ring_rows), bar = full0 + 8 * st;
    const uint32_t to = ring0 + st * 4 * row_bytes;
    mbar_arrive_expect_tx(bar, row_bytes * uint32_t((has_dx ? 2 : 0) + (has_dres ? 1 : 0) + (has_block ? 1 : 0)));
    if (has_dx) {
      bulk_load(to, resid_out + t * p.resid_out_rs, row_bytes, bar);
      bulk_load(to + row_bytes, dx + t * p.dnorm_out_rs, row_bytes, bar);
    }
    if (has_dres) bulk_load(to + 2 * row_bytes, dres + t * p.dresid_out_rs, row_bytes, bar);
    if (has_block) bulk_load(to + 3 * row_bytes, block + t * p.block_rs, row_bytes, bar);
  };
  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < p.ring_rows; ++i) mbar_init(full0 + 8 * i, 1);
    fence_barrier_init();
    for (int64_t t = row0; t < row1 && t < row0 + p.ring_rows; ++t) copy_row(t);
  }
  __syncthreads();
  start_group();
  uint32_t st = 0, phase = 0;
  int64_t t = row0;
  for (; t < row1; ++t) {
    const bool ok = mbar_wait(full0 + 8 * st, phase, &abort_flag, p.status, kStatProducerWait, p.limit_ns);
    // every thread is past the row before: its place in the ring is free
    if (!__syncthreads_and(ok)) break;
    if (tid == 0 && t > row0 && t - 1 + p.ring_rows < row1) copy_row(t - 1 + p.ring_rows);
    const T* row_r = reinterpret_cast<const T*>(ring + st * 4 * row_bytes);
    const T *row_x = row_r + p.D, *row_d = row_x + p.D, *row_y = row_d + p.D;
    if (++st == uint32_t(p.ring_rows)) st = 0, phase ^= 1;
    if (t == group_end) {
      end_group();
      ++group;
      group_end += per;
      start_group();
    }
    uint64_t s[NV][P];
    if (has_dx) {
      uint64_t r[NV][P], x[NV][P], srr = 0, ser = 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        uint64_t w[P];
        get(true, row_r, v, r[v], 0);
        get(true, row_x, v, x[v], 0);
        get(has_pre, w_pre, v, w, one);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          srr = fma2(r[v][i], r[v][i], srr);
          ser = fma2(mul2(x[v][i], w[i]), r[v][i], ser);
        }
      }
      const float2 q = block_sum2(sum_of(srr), sum_of(ser), smem, buf);
      const float rho1 = rsqrtf(q.x * inv_d + p.eps);
      const float k1 = q.y * -inv_d * rho1 * rho1 * rho1;
      const uint64_t rho = pair_of(rho1, rho1), k = pair_of(k1, k1);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        uint64_t w[P];
        get(has_pre, w_pre, v, w, one);
        get(has_dres, row_d, v, s[v], 0);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          s[v][i] = fma2(x[v][i], mul2(w[i], rho), fma2(r[v][i], k, s[v][i]));
          s_pre[v][i] = fma2(x[v][i], mul2(r[v][i], rho), s_pre[v][i]);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v) get(has_dres, row_d, v, s[v], 0);
    }
    uint64_t y[NV][P], syy = 0, sfy = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      uint64_t f[P];
      get(has_block, row_y, v, y[v], 0);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        f[i] = mul2(scale, s[v][i]);
        syy = fma2(y[v][i], y[v][i], syy);
        sfy = fma2(mul2(s[v][i], gw[v][i]), y[v][i], sfy);
      }
      if (inside(v)) put_pairs<T>(dresid + t * p.dresid_rs + (v * nt + tid) * E, f);
    }
    if (!has_block) continue;
    uint64_t rho = one, k = 0;
    if (kPost) {
      const float2 q = block_sum2(sum_of(syy), sum_of(sfy), smem, buf);
      const float rho1 = rsqrtf(q.x * inv_d + p.eps);
      const float k1 = q.y * -inv_d * rho1 * rho1 * rho1;
      rho = pair_of(rho1, rho1);
      k = pair_of(k1, k1);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      uint64_t o[P];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        s_group[v][i] = fma2(s[v][i], kPost ? mul2(y[v][i], rho) : y[v][i], s_group[v][i]);
        o[i] = mul2(s[v][i], gw[v][i]);
        if (kPost) o[i] = fma2(y[v][i], k, mul2(rho, o[i]));
      }
      if (inside(v)) put_pairs<T>(dblock + t * p.dblock_rs + (v * nt + tid) * E, o);
    }
  }
  if (t < row1) {  // a copy did not come in time: let those on their way land
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000) {
    }
    return;
  }
  if (row0 < row1) end_group();
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * nt + tid) * E;
    if (inside(v)) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        *reinterpret_cast<uint64_t*>(part + c + 2 * i) = s_pre[v][i];
        part[p.D + c + 2 * i] = s_post[c + 2 * i];
        part[p.D + c + 2 * i + 1] = s_post[c + 2 * i + 1];
      }
    }
  }
}

// The forward direction of many wide rows, the same way: r and y through a ring, pairs of operations, the
// weights in registers.
template <typename T, int NV, bool kAll>
__global__ void __launch_bounds__(512) cconv_residual_norm_ring_kernel(const NormParams p) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ float2 smem[2][32];
  __shared__ __align__(8) uint64_t full[8];
  __shared__ int abort_flag;
  start_in_order();
  constexpr int E = 16 / int(sizeof(T)), P = E / 2;
  const T* resid = static_cast<const T*>(p.resid);  // may be resid_out
  const T* block = static_cast<const T*>(p.block);
  const T* __restrict__ gate = static_cast<const T*>(p.gate);
  const T* __restrict__ w_post = static_cast<const T*>(p.w_post);
  const T* __restrict__ w_pre = static_cast<const T*>(p.w_pre);
  T* resid_out = static_cast<T*>(p.resid_out);
  T* norm_out = static_cast<T*>(p.norm_out);
  const int nt = blockDim.x, tid = threadIdx.x;
  const bool has_block = kAll || block, has_post = kAll || w_post, has_norm = kAll || norm_out;
  auto inside = [&](int v) { return kAll || (v * nt + tid) * E < p.D; };
  const float inv_d = 1.0f / float(p.D);
  const int64_t row0 = first_row(p, blockIdx.x), row1 = first_row(p, blockIdx.x + 1);
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T;
  const uint32_t row_bytes = uint32_t(p.D) * sizeof(T), ring0 = smem_u32(ring), full0 = smem_u32(full);
  const uint64_t one = pair_of(1.0f, 1.0f), scale = pair_of(p.scale, p.scale);
  int buf = 0;
  auto get = [&](bool given, const T* from, int v, uint64_t (&f)[P], uint64_t otherwise) {
    if (given && inside(v)) {
      get_pairs<T>(from + (v * nt + tid) * E, f);
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) f[i] = otherwise;
    }
  };
  auto copy_row = [&](int64_t t) {
    const uint32_t st = uint32_t(t - row0) % uint32_t(p.ring_rows), bar = full0 + 8 * st;
    const uint32_t to = ring0 + st * 2 * row_bytes;
    mbar_arrive_expect_tx(bar, row_bytes * (has_block ? 2u : 1u));
    bulk_load(to, resid + t * p.resid_rs, row_bytes, bar);
    if (has_block) bulk_load(to + row_bytes, block + t * p.block_rs, row_bytes, bar);
  };
  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < p.ring_rows; ++i) mbar_init(full0 + 8 * i, 1);
    fence_barrier_init();
    for (int64_t t = row0; t < row1 && t < row0 + p.ring_rows; ++t) copy_row(t);
  }
  __syncthreads();
  uint64_t gw[NV][P], wpre[NV][P];  // gate * w_post of the current group; w_pre
#pragma unroll
  for (int v = 0; v < NV; ++v) get(kAll || w_pre, w_pre, v, wpre[v], one);
  int64_t group_end = row0;
  uint32_t st = 0, phase = 0;
  int64_t t = row0;
  for (; t < row1; ++t) {
    if (t == group_end || t == row0) {
      const int64_t group = t / per;
      group_end = (group + 1) * per;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        uint64_t fg[P];
        get(kAll || gate, gate + group * p.gate_rs, v, fg, one);
        get(has_post, w_post, v, gw[v], one);
#pragma unroll
        for (int i = 0; i < P; ++i) gw[v][i] = mul2(gw[v][i], fg[i]);
      }
    }
    const bool ok = mbar_wait(full0 + 8 * st, phase, &abort_flag, p.status, kStatProducerWait, p.limit_ns);
    // every thread is past the row before: its place in the ring is free
    if (!__syncthreads_and(ok)) break;
    if (tid == 0 && t > row0 && t - 1 + p.ring_rows < row1) copy_row(t - 1 + p.ring_rows);
    const T* row_r = reinterpret_cast<const T*>(ring + st * 2 * row_bytes);
    const T* row_y = row_r + p.D;
    if (++st == uint32_t(p.ring_rows)) st = 0, phase ^= 1;
    uint64_t o[NV][P], sum = 0;
    float rho1 = 1.0f;
    if (has_block) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        get(true, row_y, v, o[v], 0);
#pragma unroll
        for (int i = 0; i < P; ++i) sum = fma2(o[v][i], o[v][i], sum);
      }
      if (has_post) rho1 = rsqrtf(block_sum2(sum_of(sum), 0.0f, smem, buf).x * inv_d + p.eps);
    }
    uint64_t rho = pair_of(rho1, rho1);
    sum = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      uint64_t r[P];
      get(true, row_r, v, r, 0);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        r[i] = mul2(scale, r[i]);
        o[v][i] = has_block ? fma2(o[v][i], mul2(rho, gw[v][i]), r[i]) : r[i];
        sum = fma2(o[v][i], o[v][i], sum);
      }
      if (inside(v)) put_pairs<T>(resid_out + t * p.resid_out_rs + (v * nt + tid) * E, o[v]);
    }
    if (!has_norm) continue;
    rho1 = rsqrtf(block_sum2(sum_of(sum), 0.0f, smem, buf).x * inv_d + p.eps);
    rho = pair_of(rho1, rho1);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int i = 0; i < P; ++i) o[v][i] = mul2(o[v][i], mul2(rho, wpre[v][i]));
      if (inside(v)) put_pairs<T>(norm_out + t * p.norm_out_rs + (v * nt + tid) * E, o[v]);
    }
  }
  if (t < row1) {  // a copy did not come in time: let those on their way land
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000) {
    }
  }
}

// Rows too long for registers: column sums live in the partial table (5 rows a block here; the fifth
// holds the sums of a gate group that is complete within the block until it is written).
template <typename T>
__global__ void __launch_bounds__(512) cconv_residual_norm_backward_long_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  start_in_order();
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
  const int64_t row0 = first_row(p, blockIdx.x), row1 = first_row(p, blockIdx.x + 1);
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
      k = rho * (rho * (rho * (q.y * inv_d)));
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
      ky = rho_y * (rho_y * (rho_y * (q.y * inv_d)));
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
// i end in, if block i is the first that it lies in.  32 x V columns by 16 slices of the table a block, 8 loads
// of V numbers a thread at a time: the table (16384 x 4096 with 8 gates: 15 MB) is read in three rounds of
// latency, 7 us; with loads of one number, 4 at a time, it took 14 us.
template <typename T, int V>
__global__ void __launch_bounds__(512) cconv_residual_norm_sums_kernel(const NormParams p) {
  struct __align__(V * 4) Vec {
    float v[V];
    __device__ __forceinline__ void add(const Vec& o) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += o.v[i];
    }
  };
  __shared__ Vec smem[16][32];
  start_in_order();
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * V;
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T;
  int b0 = 0, b1 = p.nb - 1, slot = int(blockIdx.y);
  T* to = static_cast<T*>(blockIdx.y == 0 ? p.dw_pre : p.dw_post);
  int64_t group = 0;
  if (blockIdx.y >= 2) {
    // every block has a row (nb <= T); row t lies in block ceil((t + 1) nb / T) - 1
    const int i = int(blockIdx.y) - 2;
    group = p.sums_by_group ? i : (first_row(p, i + 1) - 1) / per;
    const int64_t g0 = group * per, g1 = g0 + per < p.T ? g0 + per : p.T;
    b0 = int(((g0 + 1) * p.nb + p.T - 1) / p.T) - 1;
    b1 = int((g1 * p.nb + p.T - 1) / p.T) - 1;
    if (b0 == b1 || (!p.sums_by_group && b0 != i)) return;  // complete already; another block's
    to = static_cast<T*>(p.dgate) + group * p.dgate_rs;
  } else if (!to) {
    return;
  }
  Vec s = {};
  if (c < p.D) {
    const float* from = p.part + int64_t(slot) * p.D + c;
    const int64_t step = 4 * int64_t(p.D);
    auto load = [&](const float* at) { return *reinterpret_cast<const Vec*>(at); };
    if (blockIdx.y >= 2) {
      // the group's rows are the last group of its first block and the first of the others, unless they
      // begin that block
      const bool last = first_row(p, b0) / per != group;
      from = p.part + 2 * int64_t(p.D) + c;
      if (last && slice == 0) s = load(from + b0 * step + p.D);
      b0 += last;
    }
    for (int b = b0 + slice; b <= b1; b += 128) {
      Vec v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = b + 16 * i <= b1 ? load(from + (b + 16 * i) * step) : Vec{};
#pragma unroll
      for (int w = 4; w; w /= 2)
#pragma unroll
        for (int i = 0; i < w; ++i) v[i].add(v[i + w]);
      s.add(v[0]);
    }
  }
  smem[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && c < p.D) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s.add(smem[i][lane]);
#pragma unroll
    for (int i = 0; i < V; ++i) to[c + i] = from_f32<T>(s.v[i]);
  }
}

// Shared memory of an SM for the rings of the backward blocks on it, and what a block has besides (its own
// few KB, and the sums of dw_post).
constexpr int64_t kRingSmem = 216 * 1024, kRingOwn = 2048;
int64_t ring_rows(int64_t D, int es, int64_t blocks) {
  return (kRingSmem / blocks / 1024 * 1024 - kRingOwn - 4 * D) / (4 * D * es);
}
// Backward blocks that share an SM: about 512 threads of 16 elements, so that one block's row covers the
// other's reductions while the table of partial sums stays small against the arrays (at D = 4096, bf16:
// two blocks of 256 threads; with 8 elements a thread, two blocks of 512, it took 1.4 times as long); fewer where a
// ring of each would not hold two rows.
int64_t blocks_an_sm(int64_t D, int es) {
  const int64_t threads = std::max<int64_t>(32, std::min<int64_t>(512, round_up64(cdiv64(D, 16), 32)));
  int64_t n = std::min<int64_t>(16, 512 / threads);
  while (n > 1 && ring_rows(D, es, n) < 2) --n;
  return n;
}

// Threads a block and accesses a thread for rows of D elements taken E at a time: at most `held`
// elements a thread, whole warps, one access a thread as long as that leaves `few` threads or fewer.
struct Shape {
  int threads, nv;
};
Shape shape_of(int64_t D, int E, int held, int most, int few = 256) {
  const int64_t acc = cdiv64(D, E);
  int nv = 1;
  while (nv * E < held && acc > int64_t(nv) * few) nv *= 2;
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

template <typename F>
cudaError_t allow_ring(F f, bool (&ready)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!__atomic_load_n(&ready[dev & 63], __ATOMIC_ACQUIRE)) {
    e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kRingSmem));
    if (e != cudaSuccess) return e;
    __atomic_store_n(&ready[dev & 63], true, __ATOMIC_RELEASE);
  }
  return cudaSuccess;
}

template <typename T, int E, int NV>
cudaError_t launch_forward_nv(const NormParams& p, int threads, int64_t grid, cudaStream_t s) {
  return launch(cconv_residual_norm_kernel<T, E, NV>, dim3(unsigned(grid)), threads, 0, 1, s, p);
}

template <typename T, int NV, bool kAll>
cudaError_t launch_forward_ring(const NormParams& p, int threads, cudaStream_t s) {
  auto f = cconv_residual_norm_ring_kernel<T, NV, kAll>;
  static bool ready[64] = {};
  const cudaError_t e = allow_ring(f, ready);
  if (e != cudaSuccess) return e;
  return launch(f, dim3(unsigned(p.nb)), threads, size_t(p.D) * p.ring_rows * 2 * sizeof(T), 1, s, p);
}

// Shared memory of a row of one array in the ring of rows that begin anywhere.
int64_t narrow_slot(int64_t row_bytes) { return round_up64(row_bytes, 16) + 16; }
// Threads and elements a thread there: 64 to 512 threads, 12 or 16 elements (8 where D is at most 512).
Shape narrow_shape(int64_t D) {
  if (D <= 512) return {64, 8};
  for (int threads = 64; threads <= 512; threads *= 2) {
    if (D <= threads * 12) return {threads, 12};
    if (D <= threads * 16) return {threads, 16};
  }
  return {0, 0};
}
// Calls f with the shape's numbers as constants: f(elements, threads).
template <typename F>
cudaError_t with_narrow_shape(const Shape& n, F f) {
  auto elements = [&](auto threads) {
    if (n.nv == 12) return f(std::integral_constant<int, 12>(), threads);
    return f(std::integral_constant<int, 16>(), threads);
  };
  if (n.nv == 8) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 64>());
  if (n.threads == 64) return elements(std::integral_constant<int, 64>());
  if (n.threads == 128) return elements(std::integral_constant<int, 128>());
  if (n.threads == 256) return elements(std::integral_constant<int, 256>());
  return elements(std::integral_constant<int, 512>());
}
// Whether the rows of an array can go through it: none but the first and last touch its ends.
bool narrow_fits(const void* q, int64_t rs, const NormParams& p, int es) {
  return !q || (rs * es >= 16 && p.D * es >= 64);
}

template <typename T>
cudaError_t launch_forward(NormParams p, int sms, cudaStream_t s) {
  constexpr int kWide = 16 / int(sizeof(T)), kMost = 16 / kWide;
  const bool w = wide(p, sizeof(T), false);
  const Shape sh = shape_of(p.D, w ? kWide : 1, 16, 1024);
  const int threads = sh.threads ? sh.threads : 1024;
  // Many wide rows: blocks of about 1024 threads an SM go through rows of their own, fewer where their rings
  // would not hold two rows each.
  int64_t an_sm = std::max(1, std::min(16, 1024 / threads));
  auto rows = [&](int64_t blocks) { return (kRingSmem / blocks / 1024 * 1024 - kRingOwn) / (2 * p.D * int64_t(sizeof(T))); };
  while (an_sm > 1 && rows(an_sm) < 2) --an_sm;
  if (w && sh.threads && sh.threads <= 512 && rows(an_sm) >= 2 && p.T >= 4 * an_sm * sms) {
    p.nb = int(an_sm * sms);
    p.ring_rows = int(std::min<int64_t>(8, rows(an_sm)));
    const bool all = p.block && p.w_post && p.w_pre && p.gate && p.norm_out && p.D == int64_t(sh.threads) * sh.nv * kWide;
    if (sh.nv == 1) return all ? launch_forward_ring<T, 1, true>(p, threads, s) : launch_forward_ring<T, 1, false>(p, threads, s);
    if (sh.nv == 2) return all ? launch_forward_ring<T, 2, true>(p, threads, s) : launch_forward_ring<T, 2, false>(p, threads, s);
    return all ? launch_forward_ring<T, kMost, true>(p, threads, s) : launch_forward_ring<T, kMost, false>(p, threads, s);
  }
  const int64_t grid = std::min<int64_t>(p.T, int64_t(sms) * std::max(1, std::min(32, 1024 / threads)));
  if (!sh.threads) return launch(cconv_residual_norm_long_kernel<T>, dim3(unsigned(grid)), threads, 0, 1, s, p);
  if (w) {
    if (sh.nv == 1) return launch_forward_nv<T, kWide, 1>(p, threads, grid, s);
    if (sh.nv == 2) return launch_forward_nv<T, kWide, 2>(p, threads, grid, s);
    return launch_forward_nv<T, kWide, kMost>(p, threads, grid, s);
  }
  // many rows that are not wide: the same with their own ring
  const Shape n = narrow_shape(p.D);
  if (n.threads && narrow_fits(p.resid, p.resid_rs, p, sizeof(T)) && narrow_fits(p.block, p.block_rs, p, sizeof(T))) {
    const int64_t es = sizeof(T), slot = narrow_slot(p.D * es), spare = n.threads * n.nv * es;
    an_sm = 1024 / n.threads;
    auto narrow_rows = [&](int64_t blocks) { return (kRingSmem / blocks / 1024 * 1024 - kRingOwn - spare) / (2 * slot); };
    while (an_sm > 1 && narrow_rows(an_sm) < 2) --an_sm;
    if (narrow_rows(an_sm) >= 2 && p.T >= 4 * an_sm * sms) {
      p.nb = int(an_sm * sms);
      p.ring_rows = int(std::min<int64_t>(8, narrow_rows(an_sm)));
      p.ring_slot = uint32_t(slot);
      return with_narrow_shape(n, [&](auto nv, auto nt) {
        auto f = cconv_residual_norm_narrow_kernel<T, decltype(nv)::value, decltype(nt)::value>;
        static bool ready[64] = {};
        const cudaError_t e = allow_ring(f, ready);
        if (e != cudaSuccess) return e;
        return launch(f, dim3(unsigned(p.nb)), nt, size_t(p.ring_rows) * 2 * slot + spare, 1, s, p);
      });
    }
  }
  if (sh.nv == 1) return launch_forward_nv<T, 1, 1>(p, threads, grid, s);
  if (sh.nv == 2) return launch_forward_nv<T, 1, 2>(p, threads, grid, s);
  if (sh.nv == 4) return launch_forward_nv<T, 1, 4>(p, threads, grid, s);
  if (sh.nv == 8) return launch_forward_nv<T, 1, 8>(p, threads, grid, s);
  return launch_forward_nv<T, 1, 16>(p, threads, grid, s);
}

template <typename T, int NV, bool kAll, bool kPost>
cudaError_t launch_ring_as(NormParams p, int threads, cudaStream_t s) {
  auto f = cconv_residual_norm_backward_ring_kernel<T, NV, kAll, kPost>;
  static bool ready[64] = {};
  const cudaError_t e = allow_ring(f, ready);
  if (e != cudaSuccess) return e;
  p.ring_rows = int(std::min<int64_t>(8, ring_rows(p.D, sizeof(T), blocks_an_sm(p.D, sizeof(T)))));
  return launch(f, dim3(unsigned(p.nb)), threads, size_t(p.D) * (size_t(p.ring_rows) * 4 * sizeof(T) + 4), 1, s, p);
}

template <typename T, int NV>
cudaError_t launch_ring(const NormParams& p, bool all, int threads, cudaStream_t s) {
  if (all) return launch_ring_as<T, NV, true, true>(p, threads, s);
  return p.w_post ? launch_ring_as<T, NV, false, true>(p, threads, s) : launch_ring_as<T, NV, false, false>(p, threads, s);
}

template <typename T, int NV>
cudaError_t launch_plain(const NormParams& p, int threads, cudaStream_t s) {
  return launch(cconv_residual_norm_backward_kernel<T, NV, 0>, dim3(unsigned(p.nb)), threads, 0, 1, s, p);
}

// The same with rows through the ring, where they are many and it has room: fewer blocks then, if need be.
template <typename T>
bool use_narrow_ring(NormParams* p, Shape* n) {
  const int64_t es = sizeof(T), slot = narrow_slot(p->D * es);
  *n = narrow_shape(p->D);
  if (!n->threads) return false;
  const int64_t an_sm = 512 / n->threads, spare = n->threads * n->nv * es;  // w_pre, and what lies behind the last row
  const int64_t rows = (kRingSmem / an_sm / 1024 * 1024 - kRingOwn - spare) / (4 * slot);
  if (p->T < 4 * int64_t(p->nb) || rows < 2 || !narrow_fits(p->dnorm_out, p->dnorm_out_rs, *p, es) ||
      !narrow_fits(p->dnorm_out ? p->resid_out : nullptr, p->resid_out_rs, *p, es) ||
      !narrow_fits(p->dresid_out, p->dresid_out_rs, *p, es) || !narrow_fits(p->block, p->block_rs, *p, es))
    return false;
  p->nb = int(std::min<int64_t>(p->nb, std::max<int64_t>(1, p->nb * an_sm / blocks_an_sm(p->D, es))));
  p->ring_rows = int(std::min<int64_t>(8, rows));
  p->ring_slot = uint32_t(slot);
  return true;
}

// Rows of more than 8192: 512 threads a block, 12 or 16 columns a thread, which a block must have at least 8 or 12 of
// (Across::kSure), and a ring of two rows.  Not every SM finds others for a cluster of more than 2.
template <typename T>
bool use_cluster(NormParams* p, Shape* n) {
  const int64_t es = sizeof(T);
  if (p->T < 2 || !narrow_fits(p->dnorm_out, p->dnorm_out_rs, *p, es) ||
      !narrow_fits(p->dnorm_out ? p->resid_out : nullptr, p->resid_out_rs, *p, es) ||
      !narrow_fits(p->dresid_out, p->dresid_out_rs, *p, es) || !narrow_fits(p->block, p->block_rs, *p, es))
    return false;
  for (int parts = 2; parts <= kMostParts; parts *= 2) {
    const int64_t columns = cdiv64(p->D, parts), slot = narrow_slot(columns * es);
    const int nv = columns <= 512 * 12 ? 12 : 16;
    const int64_t rows = (kRingSmem - kRingOwn - 512 * nv * es) / (4 * slot);
    if (columns > 512 * 16 || p->D / parts < 512 * (nv - 4) || rows < 2) continue;
    *n = {512, nv};
    p->parts = parts;
    p->nb = std::max(1, parts == 2 ? p->nb / 2 : p->nb * 5 / (6 * parts));
    p->ring_rows = int(std::min<int64_t>(8, rows));
    p->ring_slot = uint32_t(slot);
    return true;
  }
  return false;
}

template <typename T>
cudaError_t launch_backward(NormParams p, cudaStream_t s) {
  constexpr int kWide = 16 / int(sizeof(T));
  const bool w = wide(p, sizeof(T), true) && ring_rows(p.D, sizeof(T), blocks_an_sm(p.D, sizeof(T))) >= 2;
  // Many wide rows: all of 16 elements a thread, for which blocks_an_sm counts (16384 x 1000 bf16: 64 us, with
  // 8 elements, of whose blocks not all fit, 73 us).
  const Shape sh = shape_of(p.D, w ? kWide : 1, 16, 512, w && p.T >= 4 * int64_t(p.nb) ? 32 : 256);
  const bool all = p.dnorm_out && p.dresid_out && p.block && p.w_pre && p.w_post && p.gate &&
                   p.D == int64_t(sh.threads) * sh.nv * kWide;
  cudaError_t e = cudaSuccess;
  Shape n;
  if (!sh.threads && use_cluster<T>(&p, &n)) {
    auto run = [&](auto nv) {
      auto f = cconv_residual_norm_backward_kernel<T, decltype(nv)::value, 512, true>;
      static bool ready[64] = {};
      const cudaError_t e = allow_ring(f, ready);
      if (e != cudaSuccess) return e;
      return launch(f, dim3(unsigned(p.nb * p.parts)), 512, size_t(p.ring_rows) * 4 * p.ring_slot + 512 * nv * sizeof(T), p.parts,
                    s, p);
    };
    e = n.nv == 12 ? run(std::integral_constant<int, 12>()) : run(std::integral_constant<int, 16>());
  } else if (!w && use_narrow_ring<T>(&p, &n)) {
    e = with_narrow_shape(n, [&](auto nv, auto nt) {
      auto f = cconv_residual_norm_backward_kernel<T, decltype(nv)::value, decltype(nt)::value>;
      static bool ready[64] = {};
      const cudaError_t e = allow_ring(f, ready);
      if (e != cudaSuccess) return e;
      return launch(f, dim3(unsigned(p.nb)), nt, size_t(p.ring_rows) * 4 * p.ring_slot + nt * nv * sizeof(T), 1, s, p);
    });
  } else if (!sh.threads) {
    e = launch(cconv_residual_norm_backward_long_kernel<T>, dim3(unsigned(p.nb)), 512, 0, 1, s, p);
  } else if (w) {
    constexpr int kMost = 16 / kWide;
    if (sh.nv == 1) e = launch_ring<T, 1>(p, all, sh.threads, s);
    else if (sh.nv == 2) e = launch_ring<T, 2>(p, all, sh.threads, s);
    else e = launch_ring<T, kMost>(p, all, sh.threads, s);
  } else {
    if (sh.nv == 1) e = launch_plain<T, 1>(p, sh.threads, s);
    else if (sh.nv == 2) e = launch_plain<T, 2>(p, sh.threads, s);
    else if (sh.nv == 4) e = launch_plain<T, 4>(p, sh.threads, s);
    else if (sh.nv == 8) e = launch_plain<T, 8>(p, sh.threads, s);
    else e = launch_plain<T, 16>(p, sh.threads, s);
  }
  if (e != cudaSuccess) return e;
  NormParams q = p;
  const int64_t per = p.rows_per_gate ? p.rows_per_gate : p.T, groups = cdiv64(p.T, per);
  q.sums_by_group = groups <= p.nb;
  const int64_t items = !p.gate || per == 1 ? 0 : q.sums_by_group ? groups : p.nb - 1;
  const int V = p.D % 4 ? 1 : 4;
  const dim3 grid(unsigned(cdiv64(p.D, 32 * V)), unsigned(2 + items));
  if (V == 4) return launch(cconv_residual_norm_sums_kernel<T, 4>, grid, 512, 0, 1, s, q);
  return launch(cconv_residual_norm_sums_kernel<T, 1>, grid, 512, 0, 1, s, q);
}

}  // namespace

int norm_backward_blocks(int64_t T, int64_t D, int es, int sms) {
  return int(std::max<int64_t>(1, std::min<int64_t>(T, int64_t(sms) * blocks_an_sm(D, es))));
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
