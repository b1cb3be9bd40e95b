// The forward kernels of the residual norm (definitions: block_norm.cu; with 8-bit results: block_norm_quant.cu).
#pragma once
#include "block_e4m3.cuh"
#include "block_norm.cuh"

namespace cconv {
namespace {

// ---- 8-bit results ------------------------------------------------------------------------------
// The largest of |a|, |b| and |c|, NaN if one is.
__device__ __forceinline__ float largest_of(float a, float b, float c) {
  float m;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
  return m;
}

// Of elements that 128 / E neighbouring lanes hold (2 P = E each, from column c on; a row's end has zeros behind it):
// scale = max|x| / 448 of the 128 and e4m3(x / scale).  All lanes of the warp come here.  What a lane does for a block
// (scale, reciprocal) it shares among few elements, so that both quotients are formed without the division's
// instructions (16384 x 4096 bf16 with them: 113 us): Markstein's step after a product with the reciprocal, which for
// 448, a constant of 3 bits, is correctly rounded, and for x / scale within 2^-24 (1 + 2^-20).  Scales that the
// steps cannot take (and NaN) divide.
template <int P>
__device__ __forceinline__ void put_quantized(const NormParams& p, int64_t t, int c, bool inside, uint64_t (&f)[P]) {
  constexpr int kLanes = 64 / P;
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const float2 v = halves_of(f[i]);
    m = largest_of(v.x, v.y, m);
  }
  uint32_t size = size_of(m);
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) size = max(size, __shfl_xor_sync(0xffffffffu, size, o));
  if (!inside) return;  // (a warp of zeros behind the row would divide: 16384 x 5376 221 us)
  m = __uint_as_float(size);
  float scale = m * (1.0f / kMax);
  if (m > 1e-22f && m < 1e25f) {
    scale = fmaf(fmaf(scale, -kMax, m), 1.0f / kMax, scale);
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(scale));
    y = fmaf(fmaf(y, -scale, 1.0f), y, y);
    const uint64_t y2 = pair_of(y, y), minus = pair_of(-scale, -scale);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint64_t q = mul2(f[i], y2);
      f[i] = fma2(fma2(q, minus, f[i]), y2, q);
    }
  } else {
    scale = __fdiv_rn(m, kMax);
    if (scale != 0.0f) {
#pragma unroll
      for (int i = 0; i < P; ++i) f[i] = divide_pair(f[i], scale);
    }
  }
  if ((c & 127) == 0) p.q_scale[t * p.q_scale_rs + (c >> 7) * p.q_scale_cs] = scale;
  uint8_t* to = p.q + t * p.q_rs + c;
  if constexpr (P == 4) *reinterpret_cast<uint2*>(to) = make_uint2(e4m3x4(f[0], f[1]), e4m3x4(f[2], f[3]));
  else *reinterpret_cast<uint32_t*>(to) = e4m3x4(f[0], f[1]);
}

// Of a row whose element v nt + tid is the thread's (NV a thread, zeros behind the row): the maxima of 32 neighbours
// meet in shared memory, a thread for each 128 columns makes the scale and its reciprocal of them, and all take those
// (each element with divisions of its own: 16384 x 4095 bf16 435 us).
template <int kColumns>
struct AcrossScales {
  uint32_t maxima[kColumns / 32];
  float2 scale[(kColumns + 127) / 128];  // and its reciprocal, 0 where quotients are divisions
};
template <int NV, int kColumns>
__device__ __forceinline__ void put_quantized_across(const NormParams& p, int64_t t, int nt, const float (&f)[NV],
                                                     AcrossScales<kColumns>& shared) {
  const int tid = threadIdx.x, last = (p.D - 1) >> 5;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = v * nt + tid;
    const uint32_t m = __reduce_max_sync(0xffffffffu, size_of(f[v]));
    if ((tid & 31) == 0 && c < p.D) shared.maxima[c >> 5] = m;
  }
  __syncthreads();
  for (int b = tid; b * 128 < p.D; b += nt) {
    uint32_t m = shared.maxima[4 * b];
#pragma unroll
    for (int i = 1; i < 4; ++i) m = max(m, shared.maxima[min(4 * b + i, last)]);
    const float scale = __fdiv_rn(__uint_as_float(m), kMax);
    const bool quick = scale > 1e-25f && scale < 1e25f;
    shared.scale[b] = make_float2(scale, quick ? __fdiv_rn(1.0f, scale) : 0.0f);
    p.q_scale[t * p.q_scale_rs + b * p.q_scale_cs] = scale;
  }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = v * nt + tid;
    if (c >= p.D) break;
    const float2 s = shared.scale[c >> 7];
    float q = f[v] * s.y;
    q = fmaf(fmaf(q, -s.x, f[v]), s.y, q);
    if (s.y == 0.0f) q = s.x == 0.0f ? f[v] : __fdiv_rn(f[v], s.x);
    p.q[t * p.q_rs + c] = uint8_t(e4m3x4(pair_of(q, 0.0f), 0));
  }
}
template <int N>
__device__ __forceinline__ void as_pairs(const float (&f)[N], uint64_t (&o)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) o[i] = pair_of(f[2 * i], f[2 * i + 1]);
}

// A block a row (and the row gridDim.x further on, ...): few rows, whose latency counts, or rows that are not
// wide.  Everything that a row needs is asked for before its first reduction (one row of 4096: 2.5 us).
// (Without 8-bit results the sums are the first of two: with the sum of one value the compiler's code for rows that begin
// anywhere is slower, 2400 x 1001 bf16 15.6 instead of 11.2 us, 1200 x 333 5.4 instead of 4.1; elsewhere it makes no difference.)
template <typename T, int E, int NV, bool kQuant>
__global__ void __launch_bounds__(1024) cconv_residual_norm_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  __shared__ AcrossScales<kQuant && E == 1 ? NV * 1024 : 32> across;
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
  auto sum_over_block = [&](float v) { return kQuant ? block_sum1(v, smem, buf) : block_sum2(v, 0.0f, smem, buf).x; };
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
      rho = rsqrtf(sum_over_block(ss) * inv_d + p.eps);
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
    if (!kQuant && !norm_out) continue;
    rho = rsqrtf(sum_over_block(ss) * inv_d + p.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * nt + tid) * E;
      float w[E];
      vpre[v].get(w);
#pragma unroll
      for (int i = 0; i < E; ++i) o[v][i] *= w_pre ? rho * w[i] : rho;
      if (c < p.D && (!kQuant || norm_out)) V::store(norm_out + t * p.norm_out_rs + c, o[v]);
      if constexpr (kQuant && E > 1) {
        uint64_t f[E / 2];
        as_pairs(o[v], f);
        put_quantized(p, t, c, c < p.D, f);
      }
    }
    if constexpr (kQuant && E == 1) {
      float f[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) f[v] = o[v][0];
      put_quantized_across(p, t, nt, f, across);
    }
  }
}

// Rows too long for registers: the row is read again in each of the three sweeps (from L2, which sets the pace:
// nothing of a row is kept on chip but its sums, so that any length works).
template <typename T, bool kQuant>
__global__ void __launch_bounds__(1024) cconv_residual_norm_long_kernel(const NormParams p) {
  __shared__ float2 smem[2][32];
  __shared__ uint32_t maxima[2][32];
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
      rho_y = rsqrtf(block_sum1(ss, smem, buf) * inv_d + p.eps);
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
    if (kQuant || norm_out) {
      float ss = 0.0f;
      for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
        const float o = out(c);
        ss += o * o;
      }
      rho_r = rsqrtf(block_sum1(ss, smem, buf) * inv_d + p.eps);
    }
    if constexpr (kQuant) {
      // all threads take the same number of columns; a block of 128 lies within four warps of one of them
      int odd = 0;
      for (int c0 = 0; c0 < p.D; c0 += blockDim.x, odd ^= 1) {
        const int c = c0 + int(threadIdx.x), warp = threadIdx.x >> 5;
        float x = 0.0f;
        if (c < p.D) {
          const float o = out(c);
          x = w_pre ? o * rho_r * to_f32(w_pre[c]) : o * rho_r;
          resid_out[t * p.resid_out_rs + c] = from_f32<T>(o);
          if (norm_out) norm_out[t * p.norm_out_rs + c] = from_f32<T>(x);
        }
        const uint32_t m = __reduce_max_sync(0xffffffffu, size_of(x));
        if ((threadIdx.x & 31) == 0) maxima[odd][warp] = m;
        __syncthreads();
        const uint32_t* four = maxima[odd] + (warp & ~3);
        const float scale = __fdiv_rn(__uint_as_float(max(max(four[0], four[1]), max(four[2], four[3]))), kMax);
        const float q = __fdiv_rn(x, scale == 0.0f ? 1.0f : scale);
        if (c < p.D) {
          p.q[t * p.q_rs + c] = uint8_t(e4m3x4(pair_of(q, 0.0f), 0));
          if ((c & 127) == 0) p.q_scale[t * p.q_scale_rs + (c >> 7) * p.q_scale_cs] = scale;
        }
      }
      __syncthreads();  // the next row's maxima come after these have been read
    } else {
      for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
        const float o = out(c);
        resid_out[t * p.resid_out_rs + c] = from_f32<T>(o);
        if (norm_out) norm_out[t * p.norm_out_rs + c] = from_f32<T>(w_pre ? o * rho_r * to_f32(w_pre[c]) : o * rho_r);
      }
    }
  }
}

// Many rows that are not wide, through a ring for rows that begin anywhere (16384 x 4095 bf16: 127 us, 224 with a block size known at
// the launch; with a block a row and everything from global memory 516 us).
// (Blocks an SM that the compiler keeps registers for: without 8-bit results none are named.  Naming one is no lower
// limit but leave to take 104 to 131 registers instead of 72 to 109: 16384 x 4095 192 us, 16384 x 2047 76 instead of 62.)
constexpr int narrow_threads(int nv) { return nv == 8 ? 1024 : 512; }  // of an SM, of 8-bit results
template <typename T, int NV, int kThreads, bool kQuant>
__global__ void __launch_bounds__(kThreads, kQuant ? narrow_threads(NV) / kThreads : 0) cconv_residual_norm_narrow_kernel(const NormParams p) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ AcrossScales<kQuant ? NV * kThreads : 32> across;
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
      rho = rsqrtf(block_sum1(ss, smem, buf) * inv_d + p.eps);
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
    if (!kQuant && !norm_out) continue;
    rho = rsqrtf(block_sum1(ss, smem, buf) * inv_d + p.eps);
    to = norm_out + t * p.norm_out_rs;
    if (!kQuant || norm_out) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (A::inside(v, p.D)) to[A::column(v)] = from_f32<T>(o[v] * (rho * wpre[v]));
    }
    if constexpr (kQuant) {
#pragma unroll
      for (int v = 0; v < NV; ++v) o[v] = A::inside(v, p.D) ? o[v] * (rho * wpre[v]) : 0.0f;
      put_quantized_across(p, t, kThreads, o, across);
    }
  }
  if (t < row1) {  // a copy did not come in time: let those on their way land
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000) {
    }
  }
}

// The forward direction of many wide rows, the same way: r and y through a ring, pairs of operations, the
// weights in registers.
// (8-bit results: the registers that 1024 threads of an SM may have.  Others take up to 84, or with kRoomy, for blocks of
// at most 256 threads of which two share an SM all the same, up to 96: 16384 x 4080 bf16 89 instead of 99 us, 8192 x 2048
// fp32 47.4 instead of 48.6; where every access lies in the row of 16-bit elements they do not pay, 16384 x 4096 94 instead
// of 92, and larger blocks would lose their neighbour, 16384 x 5376 154 instead of 135.)
// kAll: every operand is there; kExact: and every access of every thread lies in the row.
template <typename T, int NV, bool kAll, bool kExact, bool kRoomy, bool kQuant>
__global__ void __launch_bounds__(kRoomy ? 256 : 512, kQuant || kRoomy ? 2 : 0) cconv_residual_norm_ring_kernel(const NormParams p) {
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
  const bool has_block = kAll || block, has_post = kAll || w_post, has_norm = (kAll && !kQuant) || norm_out;
  auto inside = [&](int v) { return kExact || (v * nt + tid) * E < p.D; };
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
      if (has_post) rho1 = rsqrtf(block_sum1(sum_of(sum), smem, buf) * inv_d + p.eps);
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
    if (!kQuant && !has_norm) continue;
    rho1 = rsqrtf(block_sum1(sum_of(sum), smem, buf) * inv_d + p.eps);
    rho = pair_of(rho1, rho1);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int i = 0; i < P; ++i) o[v][i] = mul2(o[v][i], mul2(rho, wpre[v][i]));
      const int c = (v * nt + tid) * E;
      if ((!kQuant || has_norm) && inside(v)) put_pairs<T>(norm_out + t * p.norm_out_rs + c, o[v]);
      if constexpr (kQuant) put_quantized(p, t, c, inside(v), o[v]);
    }
  }
  if (t < row1) {  // a copy did not come in time: let those on their way land
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000) {
    }
  }
}

template <typename T, int E, int NV, bool kQuant>
cudaError_t launch_forward_nv(const NormParams& p, int threads, int64_t grid, cudaStream_t s) {
  return launch(cconv_residual_norm_kernel<T, E, NV, kQuant>, dim3(unsigned(grid)), threads, 0, 1, s, p);
}

template <typename T, int NV, bool kAll, bool kExact, bool kRoomy, bool kQuant>
cudaError_t launch_forward_ring_as(const NormParams& p, int threads, cudaStream_t s) {
  auto f = cconv_residual_norm_ring_kernel<T, NV, kAll, kExact, kRoomy, kQuant>;
  static bool ready[64] = {};
  const cudaError_t e = allow_ring(f, ready);
  if (e != cudaSuccess) return e;
  return launch(f, dim3(unsigned(p.nb)), threads, size_t(p.D) * p.ring_rows * 2 * sizeof(T), 1, s, p);
}

template <typename T, int NV, bool kQuant>
cudaError_t launch_forward_ring(const NormParams& p, int threads, cudaStream_t s) {
  const bool all = p.block && p.w_post && p.w_pre && p.gate && (kQuant || p.norm_out);
  if (!all) return launch_forward_ring_as<T, NV, false, false, false, kQuant>(p, threads, s);
  const bool exact = p.D * int64_t(sizeof(T)) == int64_t(threads) * NV * 16;
  // more than 256 threads come with 16 elements a thread alone
  constexpr bool kMayBeLarge = kQuant || NV * 16 / int(sizeof(T)) == 16, kRoomyExact = !kQuant && sizeof(T) == 4;
  if constexpr (kMayBeLarge) {
    if (kQuant || threads > 256)
      return exact ? launch_forward_ring_as<T, NV, true, true, false, kQuant>(p, threads, s)
                   : launch_forward_ring_as<T, NV, true, false, false, kQuant>(p, threads, s);
  }
  if constexpr (!kQuant) {
    if (!exact) return launch_forward_ring_as<T, NV, true, false, true, kQuant>(p, threads, s);
    return launch_forward_ring_as<T, NV, true, true, kRoomyExact, kQuant>(p, threads, s);
  }
}

template <typename T, bool kQuant>
cudaError_t launch_forward(NormParams p, int sms, cudaStream_t s) {
  constexpr int kWide = 16 / int(sizeof(T)), kMost = 16 / kWide;
  // (of 8-bit results a lane writes kWide bytes)
  const bool w = wide(p, sizeof(T), false) && (!kQuant || ((reinterpret_cast<uintptr_t>(p.q) | uintptr_t(p.q_rs)) & (kWide - 1)) == 0);
  const Shape sh = shape_of(p.D, w ? kWide : 1, 16, 1024);
  const int threads = sh.threads ? sh.threads : 1024;
  // Many wide rows: blocks of about 1024 threads an SM go through rows of their own, fewer where their rings
  // would not hold two rows each.
  int64_t an_sm = std::max(1, std::min(16, 1024 / threads));
  auto rows = [&](int64_t blocks) { return (kRingSmem / blocks / 1024 * 1024 - kRingOwn) / (2 * p.D * int64_t(sizeof(T))); };
  while (an_sm > 1 && rows(an_sm) < 2) --an_sm;
  // (8-bit results of long rows from a row a block on: 700 x 4096 9.4 us, a block a row 11.1; 1184 x 1000 4.9 and 3.9)
  const int least = kQuant && sh.nv > 1 ? 1 : 4;
  if (w && sh.threads && sh.threads <= 512 && rows(an_sm) >= 2 && p.T >= least * an_sm * sms) {
    p.nb = int(an_sm * sms);
    p.ring_rows = int(std::min<int64_t>(8, rows(an_sm)));
    if (sh.nv == 1) return launch_forward_ring<T, 1, kQuant>(p, threads, s);
    if (sh.nv == 2) return launch_forward_ring<T, 2, kQuant>(p, threads, s);
    return launch_forward_ring<T, kMost, kQuant>(p, threads, s);
  }
  const int64_t grid = std::min<int64_t>(p.T, int64_t(sms) * std::max(1, std::min(32, 1024 / threads)));
  if (!sh.threads) return launch(cconv_residual_norm_long_kernel<T, kQuant>, dim3(unsigned(grid)), threads, 0, 1, s, p);
  if (w) {
    if (sh.nv == 1) return launch_forward_nv<T, kWide, 1, kQuant>(p, threads, grid, s);
    if (sh.nv == 2) return launch_forward_nv<T, kWide, 2, kQuant>(p, threads, grid, s);
    return launch_forward_nv<T, kWide, kMost, kQuant>(p, threads, grid, s);
  }
  // many rows that are not wide: the same with their own ring
  const Shape n = kQuant ? narrow_quant_shape(p.D) : narrow_shape(p.D);
  if (n.threads && narrow_fits(p.resid, p.resid_rs, p, sizeof(T)) && narrow_fits(p.block, p.block_rs, p, sizeof(T))) {
    const int64_t es = sizeof(T), slot = narrow_slot(p.D * es), spare = n.threads * n.nv * es;
    an_sm = (kQuant ? narrow_threads(n.nv) : 1024) / n.threads;
    auto narrow_rows = [&](int64_t blocks) { return (kRingSmem / blocks / 1024 * 1024 - kRingOwn - spare) / (2 * slot); };
    while (an_sm > 1 && narrow_rows(an_sm) < 2) --an_sm;
    if (narrow_rows(an_sm) >= 2 && p.T >= 4 * an_sm * sms) {
      p.nb = int(an_sm * sms);
      p.ring_rows = int(std::min<int64_t>(8, narrow_rows(an_sm)));
      p.ring_slot = uint32_t(slot);
      auto go = [&](auto nv, auto nt) {
        auto f = cconv_residual_norm_narrow_kernel<T, decltype(nv)::value, decltype(nt)::value, kQuant>;
        static bool ready[64] = {};
        const cudaError_t e = allow_ring(f, ready);
        if (e != cudaSuccess) return e;
        return launch(f, dim3(unsigned(p.nb)), nt, size_t(p.ring_rows) * 2 * slot + spare, 1, s, p);
      };
      if constexpr (kQuant) return with_narrow_quant_shape(n, go);
      else return with_narrow_shape(n, go);
    }
  }
  if (sh.nv == 1) return launch_forward_nv<T, 1, 1, kQuant>(p, threads, grid, s);
  if (sh.nv == 2) return launch_forward_nv<T, 1, 2, kQuant>(p, threads, grid, s);
  if (sh.nv == 4) return launch_forward_nv<T, 1, 4, kQuant>(p, threads, grid, s);
  if (sh.nv == 8) return launch_forward_nv<T, 1, 8, kQuant>(p, threads, grid, s);
  return launch_forward_nv<T, 1, 16, kQuant>(p, threads, grid, s);
}

}  // namespace
}  // namespace cconv
