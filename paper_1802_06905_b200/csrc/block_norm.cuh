// What the kernels of the residual norm share: rows in registers and in shared memory, their sums and launch shapes.
#pragma once
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

// The same of one value.
__device__ __forceinline__ float block_sum1(float a, float2 (*smem)[32], int& buf) {
  a = warp_sum(a);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return a;
  float* const sums = reinterpret_cast<float*>(smem[buf]);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = a;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  buf ^= 1;
  return warp_sum(lane < warps ? sums[lane] : 0.0f);
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
  static constexpr int kSure = kThreads && NV > 8 ? NV - 4 : kThreads > 64 ? NV / 2 : 0;  // elements that every thread has
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

// Shared memory of an SM for the rings of the backward blocks on it, and what a block has besides (its own
// few KB, and the sums of dw_post).
constexpr int64_t kRingSmem = 216 * 1024, kRingOwn = 2048;
inline int64_t ring_rows(int64_t D, int es, int64_t blocks) {
  return (kRingSmem / blocks / 1024 * 1024 - kRingOwn - 4 * D) / (4 * D * es);
}
// Backward blocks that share an SM: about 512 threads of 16 elements, so that one block's row covers the
// other's reductions while the table of partial sums stays small against the arrays (at D = 4096, bf16:
// two blocks of 256 threads; with 8 elements a thread, two blocks of 512, it took 1.4 times as long); fewer where a
// ring of each would not hold two rows.
inline int64_t blocks_an_sm(int64_t D, int es) {
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
inline Shape shape_of(int64_t D, int E, int held, int most, int few = 256) {
  const int64_t acc = cdiv64(D, E);
  int nv = 1;
  while (nv * E < held && acc > int64_t(nv) * few) nv *= 2;
  const int64_t threads = round_up64(cdiv64(acc, nv), 32);
  return threads <= most ? Shape{int(threads), nv} : Shape{0, 0};
}

inline bool wide(const NormParams& p, int es, bool backward) {
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

// Shared memory of a row of one array in the ring of rows that begin anywhere.
inline int64_t narrow_slot(int64_t row_bytes) { return round_up64(row_bytes, 16) + 16; }
// Threads and elements a thread there: 64 to 512 threads, 12 or 16 elements (8 where D is at most 512).
inline Shape narrow_shape(int64_t D) {
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
// The same for 8-bit results: 8 elements a thread as long as that is enough, so that 1024 threads share an SM.
inline Shape narrow_quant_shape(int64_t D) {
  for (int threads : {64, 128, 192, 256, 384, 512})
    if (D <= threads * 8) return {threads, 8};
  return narrow_shape(D);
}
template <typename F>
cudaError_t with_narrow_quant_shape(const Shape& n, F f) {
  auto eight = [&](auto threads) { return f(std::integral_constant<int, 8>(), threads); };
  if (n.nv == 12) return f(std::integral_constant<int, 12>(), std::integral_constant<int, 512>());
  if (n.nv == 16) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 512>());
  if (n.threads == 64) return eight(std::integral_constant<int, 64>());
  if (n.threads == 128) return eight(std::integral_constant<int, 128>());
  if (n.threads == 192) return eight(std::integral_constant<int, 192>());
  if (n.threads == 256) return eight(std::integral_constant<int, 256>());
  if (n.threads == 384) return eight(std::integral_constant<int, 384>());
  return eight(std::integral_constant<int, 512>());
}
// Whether the rows of an array can go through it: none but the first and last touch its ends.
inline bool narrow_fits(const void* q, int64_t rs, const NormParams& p, int es) {
  return !q || (rs * es >= 16 && p.D * es >= 64);
}

}  // namespace
}  // namespace cconv
