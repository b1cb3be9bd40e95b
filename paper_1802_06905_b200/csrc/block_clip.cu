// The norm over all elements of a list of gradients, and their clipping.
//
//   norm = sqrt(sum of squares),  factor = min(1, max_norm / (norm + eps)),  out = factor gradient
//
// Two passes, since the factor needs every element: the first reads and leaves a partial sum a block, the
// second adds those up (every block of its first launch for itself, in a fixed order; where tensors are so many that
// there are more launches, those read the norm that the first has left), reads again and writes.  Both are bound by HBM.  The
// second goes through each block's share backwards, so that what the first read last comes out of L2.
// Where nothing is to be done in place (factor 1) the second pass ends after the sums.
//
// Squares are added up in fp32 over the 16 to 64 elements that a thread has of a piece, which go on in 64 bits.  Where
// fp32 cannot hold them (elements beyond 1e18, or all below 1e-15) the elements are squared in 64 bits.
#include "block_clip.h"

#include <algorithm>

#include "block_device.cuh"
#include "block_launch.h"

namespace cconv {
namespace {

constexpr int kThreads = 256, kBlocksAnSm = 4;

// A tensor as rows of elements.  Pieces are kVectors x 16 bytes a thread of a row or, where rows are short or elements
// apart (`scattered`), as many elements in the order of rows.
struct Item {
  const void* p;
  void* out;
  int64_t rows, cols, rs, cs, out_rs, out_cs, row_pieces;
  int64_t first;  // its first piece among those of the launch
  int32_t dtype, scattered;
};
template <int N>
struct Table {
  int64_t pieces;
  int count;
  Item item[N];
};
struct ClipParams {
  double* sums;    // partial sums of squares
  int blocks;      // of them; 0: the norm is there already
  float* norm;
  float max_norm, eps;
  int in_place;
};

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double smem[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) s += smem[i];
  return s;
}

// What a thread has of a piece: up to kVectors accesses of 16 bytes, and one element in front of and behind them.
template <typename T>
struct Piece {
  static constexpr int E = 16 / int(sizeof(T));
  const T* from;
  int head, vectors, tail;  // elements in front of the first multiple of 16 bytes, accesses, elements behind
  __device__ __forceinline__ Piece(const T* p, int64_t n) : from(p) {
    const int to_16 = int((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / int(sizeof(T));
    head = int(min(int64_t(to_16), n));
    vectors = int((n - head) / E);
    tail = int(n - head) - vectors * E;
  }
};

template <typename T>
__device__ __forceinline__ void unpack16(const uint4& w, float (&f)[16 / sizeof(T)]) {
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      f[i] = __uint_as_float(a[i]);
    } else {
      const float2 v = unpack2<T>(a[i]);
      f[2 * i] = v.x;
      f[2 * i + 1] = v.y;
    }
  }
}

// The sum of squares of what a thread has of a piece, in 64 bits where fp32 cannot hold it.
template <typename T, int kVectors>
__device__ __forceinline__ double squares(const Piece<T>& piece) {
  constexpr int E = Piece<T>::E;
  const int tid = threadIdx.x;
  const uint4* v = reinterpret_cast<const uint4*>(piece.from + piece.head);
  uint4 w[kVectors];
#pragma unroll
  for (int i = 0; i < kVectors; ++i) w[i] = i * kThreads + tid < piece.vectors ? __ldcg(v + i * kThreads + tid) : make_uint4(0, 0, 0, 0);
  float ends[2] = {0.0f, 0.0f};
  if (tid < piece.head) ends[0] = to_f32(piece.from[tid]);
  if (tid < piece.tail) ends[1] = to_f32(piece.from[piece.head + piece.vectors * E + tid]);
  float s[2] = {ends[0] * ends[0], ends[1] * ends[1]};
  uint32_t any = (__float_as_uint(ends[0]) | __float_as_uint(ends[1])) << 1;
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    float f[E];
    unpack16<T>(w[i], f);
#pragma unroll
    for (int j = 0; j < E; ++j) s[j & 1] += f[j] * f[j];
    any |= (w[i].x | w[i].y | w[i].z | w[i].w) & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu);
  }
  const float all = s[0] + s[1];
  if ((all > 1e-30f && all < 1e37f) || any == 0) return double(all);
  double exact = double(ends[0]) * double(ends[0]) + double(ends[1]) * double(ends[1]);
#pragma unroll 1
  for (int i = 0; i < kVectors; ++i) {
    if (i * kThreads + tid >= piece.vectors) break;
    float f[E];
    unpack16<T>(__ldcg(v + i * kThreads + tid), f);
#pragma unroll
    for (int j = 0; j < E; ++j) exact += double(f[j]) * double(f[j]);
  }
  return exact;
}

// The item that a piece belongs to.
template <int N>
__device__ __forceinline__ int item_of(const Table<N>& t, int64_t piece) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.item[mid].first <= piece) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

constexpr int piece_elements(int vectors, int dtype) { return kThreads * 16 * vectors / (dtype == CCONV_TYPE_FP32 ? 4 : 2); }

template <typename T, int kVectors>
__device__ __forceinline__ double item_squares(const Item& it, int64_t piece) {
  constexpr int kElements = kThreads * 16 * kVectors / int(sizeof(T));
  const T* p = static_cast<const T*>(it.p);
  if (it.scattered) {
    double s = 0.0;
    const int64_t n = it.rows * it.cols;
    for (int64_t i = piece * kElements + threadIdx.x; i < n && i < (piece + 1) * kElements; i += kThreads) {
      const double f = to_f32(p[i / it.cols * it.rs + i % it.cols * it.cs]);
      s += f * f;
    }
    return s;
  }
  const int64_t row = it.rows == 1 ? 0 : piece / it.row_pieces, c = (piece - row * it.row_pieces) * kElements;
  return squares<T, kVectors>(Piece<T>(p + row * it.rs + c, min(it.cols - c, int64_t(kElements))));
}

template <int N, int kVectors>
__global__ void __launch_bounds__(kThreads, kBlocksAnSm) cconv_square_sums_kernel(const __grid_constant__ Table<N> t, double* sums) {
  start_in_order();
  const int64_t p0 = t.pieces * blockIdx.x / gridDim.x, p1 = t.pieces * (blockIdx.x + 1) / gridDim.x;
  double s = 0.0;
  int at = item_of(t, p0);
  for (int64_t p = p0; p < p1; ++p) {
    while (at + 1 < t.count && t.item[at + 1].first <= p) ++at;
    const Item& it = t.item[at];
    if (it.dtype == CCONV_TYPE_BF16) s += item_squares<__nv_bfloat16, kVectors>(it, p - it.first);
    else if (it.dtype == CCONV_TYPE_FP16) s += item_squares<__half, kVectors>(it, p - it.first);
    else s += item_squares<float, kVectors>(it, p - it.first);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// The norm of all partial sums, the same in every thread.
__device__ __forceinline__ float norm_of(const double* sums, int n) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) s += __ldcg(sums + i);
  return float(sqrt(block_sum(s)));
}
__global__ void __launch_bounds__(kThreads) cconv_norm_of_sums_kernel(const double* sums, int n, float* norm) {
  start_in_order();
  const float v = norm_of(sums, n);
  if (threadIdx.x == 0) *norm = v;
}

template <typename T, int kVectors>
__device__ __forceinline__ void item_scale(const Item& it, int64_t piece, float by) {
  constexpr int kElements = kThreads * 16 * kVectors / int(sizeof(T)), E = 16 / int(sizeof(T));
  const T* p = static_cast<const T*>(it.p);
  T* out = static_cast<T*>(it.out);
  const int tid = threadIdx.x;
  if (it.scattered) {
    const int64_t n = it.rows * it.cols;
    for (int64_t i = piece * kElements + tid; i < n && i < (piece + 1) * kElements; i += kThreads) {
      const int64_t r = i / it.cols, c = i % it.cols;
      out[r * it.out_rs + c * it.out_cs] = from_f32<T>(by * to_f32(p[r * it.rs + c * it.cs]));
    }
    return;
  }
  const int64_t row = it.rows == 1 ? 0 : piece / it.row_pieces, c = (piece - row * it.row_pieces) * kElements;
  const Piece<T> from(p + row * it.rs + c, min(it.cols - c, int64_t(kElements)));
  T* to = out + row * it.out_rs + c;
  const uint4* v = reinterpret_cast<const uint4*>(from.from + from.head);
  uint4 w[kVectors];
#pragma unroll
  for (int i = 0; i < kVectors; ++i)
    if (i * kThreads + tid < from.vectors) w[i] = __ldcg(v + i * kThreads + tid);
  if (tid < from.head) to[tid] = from_f32<T>(by * to_f32(from.from[tid]));
  const int behind = from.head + from.vectors * E + tid;
  if (tid < from.tail) to[behind] = from_f32<T>(by * to_f32(from.from[behind]));
  to += from.head;
  const bool wide = (reinterpret_cast<uintptr_t>(to) & 15) == 0;
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const int at = i * kThreads + tid;
    if (at >= from.vectors) break;
    float f[E];
    unpack16<T>(w[i], f);
#pragma unroll
    for (int j = 0; j < E; ++j) f[j] *= by;
    if (wide) {
      uint32_t a[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) a[j] = __float_as_uint(f[j]);
        else a[j] = pack2<T>(f[2 * j], f[2 * j + 1]);
      }
      __stcs(reinterpret_cast<uint4*>(to) + at, make_uint4(a[0], a[1], a[2], a[3]));
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) to[at * E + j] = from_f32<T>(f[j]);
    }
  }
}

template <int N, int kVectors>
__global__ void __launch_bounds__(kThreads, kBlocksAnSm) cconv_clip_kernel(const __grid_constant__ Table<N> t, const ClipParams c) {
  start_in_order();
  const float norm = c.blocks ? norm_of(c.sums, c.blocks) : *c.norm;
  if (c.blocks && blockIdx.x == 0 && threadIdx.x == 0) *c.norm = norm;
  const float ratio = __fdiv_rn(c.max_norm, norm + c.eps);
  const float by = ratio >= 1.0f ? 1.0f : ratio;  // (NaN stays)
  if (by == 1.0f && c.in_place) return;
  const int64_t p0 = t.pieces * blockIdx.x / gridDim.x, p1 = t.pieces * (blockIdx.x + 1) / gridDim.x;
  if (p0 == p1) return;
  int at = item_of(t, p1 - 1);
  for (int64_t p = p1 - 1; p >= p0; --p) {
    while (t.item[at].first > p) --at;
    const Item& it = t.item[at];
    if (it.dtype == CCONV_TYPE_BF16) item_scale<__nv_bfloat16, kVectors>(it, p - it.first, by);
    else if (it.dtype == CCONV_TYPE_FP16) item_scale<__half, kVectors>(it, p - it.first, by);
    else item_scale<float, kVectors>(it, p - it.first, by);
  }
}

// ---- launches ----------------------------------------------------------------------------------
// Tables go with the launch: 40 tensors in the 4 KB that every launch has room for, 320 in the 32 KB that it may take.
constexpr int kFewItems = 40, kMostItems = 320;

int64_t pieces_of(const cconv_tensor& t, int vectors, bool scattered) {
  const int64_t n = piece_elements(vectors, t.dtype);
  return scattered ? cdiv64(t.rows * t.cols, n) : t.rows * cdiv64(t.cols, n);
}

// 8 accesses a thread and piece where there is work for all SMs all the same, else 4.
int vectors_of(const cconv_clip_args& a, int sms) {
  double bytes = 0;
  for (int64_t i = 0; i < a.count; ++i) bytes += double(a.grads[i].rows) * a.grads[i].cols * type_bytes(a.grads[i].dtype);
  return bytes >= 4.0 * sms * kBlocksAnSm * kThreads * 128 ? 8 : 4;
}

// Calls f(table, its number) for the tables of the call.
template <typename F>
int with_tables(const cconv_clip_args& a, int vectors, F f) {
  Table<kMostItems> t;
  t.count = 0;
  t.pieces = 0;
  int number = 0;
  auto send = [&]() -> cudaError_t {
    if (t.count == 0) return cudaSuccess;
    cudaError_t e;
    if (t.count <= kFewItems) {
      Table<kFewItems> few;
      few.count = t.count;
      few.pieces = t.pieces;
      std::copy(t.item, t.item + t.count, few.item);
      e = f(few, number);
    } else {
      e = f(t, number);
    }
    ++number;
    t.count = 0;
    t.pieces = 0;
    return e;
  };
  for (int64_t i = 0; i < a.count; ++i) {
    const cconv_tensor& g = a.grads[i];
    if (g.rows == 0 || g.cols == 0) continue;
    const cconv_tensor& o = a.outs ? a.outs[i] : g;
    Item& it = t.item[t.count++];
    it.p = g.data;
    it.out = o.data;
    it.rows = g.rows;
    it.cols = g.cols;
    it.rs = g.row_stride; it.cs = g.col_stride;
    it.out_rs = o.row_stride; it.out_cs = o.col_stride;
    it.dtype = g.dtype;
    it.row_pieces = cdiv64(g.cols, piece_elements(vectors, g.dtype));
    // short rows would leave most of a block idle
    it.scattered = (g.cols > 1 && (g.col_stride != 1 || o.col_stride != 1)) || (g.rows > 1 && g.cols < 1024);
    it.first = t.pieces;
    t.pieces += pieces_of(g, vectors, it.scattered);
    if (t.count == kMostItems) {
      const cudaError_t e = send();
      if (e != cudaSuccess) return block_cuda_error(e, "clipping");
    }
  }
  return block_cuda_error(send(), "clipping");
}

int blocks_of(int64_t pieces, int sms) { return int(std::min<int64_t>(pieces, int64_t(sms) * kBlocksAnSm)); }


}  // namespace

// (room for every launch's partial sums at their most)
int64_t clip_workspace(const cconv_clip_args& a, int sms) {
  return round_up64(std::max<int64_t>(1, cdiv64(a.count, kMostItems)) * sms * kBlocksAnSm * 8, 256);
}


int run_square_sums(const cconv_clip_args& a, int sms, int* sums, cudaStream_t s) {
  *sums = 0;
  double* to = static_cast<double*>(a.workspace);
  const int vectors = vectors_of(a, sms);
  return with_tables(a, vectors, [&](const auto& t, int) {
    const int n = blocks_of(t.pieces, sms);
    double* mine = to;
    to += n;
    *sums += n;
    constexpr int kItems = sizeof(t) == sizeof(Table<kFewItems>) ? kFewItems : kMostItems;
    auto go = [&](auto f) { return launch(f, dim3(unsigned(n)), kThreads, 0, 1, s, t, mine); };
    return vectors == 8 ? go(cconv_square_sums_kernel<kItems, 8>) : go(cconv_square_sums_kernel<kItems, 4>);
  });
}

int run_norm_of_sums(const cconv_clip_args& a, int sums, cudaStream_t s) {
  return block_cuda_error(launch(cconv_norm_of_sums_kernel, dim3(1), kThreads, 0, 1, s, static_cast<const double*>(a.workspace),
                                 sums, static_cast<float*>(a.norm)), "cconv_norm_of_sums_kernel");
}

int run_clip(const cconv_clip_args& a, int sms, int sums, cudaStream_t s) {
  ClipParams c{};
  c.sums = static_cast<double*>(a.workspace);
  c.norm = static_cast<float*>(a.norm);
  c.max_norm = a.max_norm;
  c.eps = a.eps;
  c.in_place = a.outs == nullptr;
  const int vectors = vectors_of(a, sms);
  return with_tables(a, vectors, [&](const auto& t, int number) {
    c.blocks = a.norm_given || number > 0 ? 0 : sums;
    const int n = blocks_of(t.pieces, sms);
    constexpr int kItems = sizeof(t) == sizeof(Table<kFewItems>) ? kFewItems : kMostItems;
    auto go = [&](auto f) { return launch(f, dim3(unsigned(n)), kThreads, 0, 1, s, t, c); };
    return vectors == 8 ? go(cconv_clip_kernel<kItems, 8>) : go(cconv_clip_kernel<kItems, 4>);
  });
}

}  // namespace cconv
