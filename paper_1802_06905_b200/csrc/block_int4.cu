// Products with weights of 4 bits and a scale for each group of 32, 64 or 128 of a row, and their quantiser.
//
//   C[m][n] = sum_g s[n][g] sum_{k in g} (q[n][k] - z[n][g]) x[m][k]
//           = sum_g s[n][g] (sum_k (16 + q) x - (16 + z) sum_k x)
//
// Few tokens: the weights are read once, into warp-wide matrix instructions; a group's sums come out of these, and are
// scaled and added up in fp32.  For one or two tokens 16 + q is the number that is multiplied: its mantissa starts with the
// four bits, so that a shift and a logical operation make two of them (6 operations for two where q - z is formed).  That
// costs a factor of 5 in the sums' rounding.  A word holds k = 0 .. 7 in its nibbles; the two that one shift brings in
// place are four apart, so x's pairs are taken four apart too.
//
// What bounds it: dependent instructions of few warps, and the two ends of a launch.  8192 x 4096, one token, 17 MB of weights:
// 7.7 to 8.2 us (2.6 at the rate of a copy), 420 instructions of a warp for 4096 weights, which would take 3 us if one were
// issued every clock; 4 warps a scheduler issue in 38 % of them.
#include "block_int4.h"

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "block_device.cuh"
#include "block_gemm.h"
#include "block_launch.h"
#include "block_mma.cuh"
#include "block_pad.h"
#include "block_steps.h"
#include "ptx_sm100.cuh"

namespace cconv {
namespace {

constexpr int kWarps = 8;

template <typename T>
struct Code;  // a nibble as the number 16 + q
template <>
struct Code<__nv_bfloat16> {
  static constexpr int kAt = 3;
  static constexpr uint32_t kMask = 0x00780078u, kBase = 0x41804180u;
};
template <>
struct Code<__half> {
  static constexpr int kAt = 6;
  static constexpr uint32_t kMask = 0x03c003c0u, kBase = 0x4c004c00u;
};
// 16 + q of nibbles i and i + 4.  `base` is kBase as a number that is not known when compiled: mask and base are then one
// operation (with two constants they are two).
template <typename T, int i>
__device__ __forceinline__ uint32_t two_of(uint32_t v, uint32_t base) {
  constexpr int kShift = Code<T>::kAt - 4 * i;
  const uint32_t at = kShift >= 0 ? v << (kShift & 31) : v >> (-kShift & 31);
  return (at & Code<T>::kMask) | base;
}

struct Int4Params {
  const char *x, *w;  // tokens by k; rows of nibbles
  int64_t x_rs, w_rs;  // bytes
  const char* w_end;   // behind the last row
  const char* scale;
  const uint8_t* zero;
  int64_t s_rs, s_cs, z_rs, z_cs;  // elements
  int64_t N;
  uint32_t x_bytes;  // of a token that may be read, a multiple of 16
  int M, scale_dtype, groups;
  uint32_t w_bytes;  // of a row
  uint32_t lies;     // bits in which rows' addresses and lengths differ from multiples of 16 bytes (of 4 they are)
  uint32_t base;     // Code<T>::kBase
  int shifted;       // rows do not all begin at multiples of 16 bytes
  int units, per;    // of 128 of k; of a warp
  Mat out;
};

__device__ __forceinline__ uint32_t load_scale(const char* p, int dtype, int64_t at) {
  if (dtype == CCONV_TYPE_FP32) return __ldg(reinterpret_cast<const uint32_t*>(p) + at);
  return __ldg(reinterpret_cast<const uint16_t*>(p) + at);
}
__device__ __forceinline__ float scale_of(uint32_t raw, int dtype) {
  if (dtype == CCONV_TYPE_FP32) return __uint_as_float(raw);
  if (dtype == CCONV_TYPE_BF16) return __uint_as_float(raw << 16);
  return __half2float(__ushort_as_half(uint16_t(raw)));
}

// kBytes of a row (from global memory, or zeros) to shared memory, not waited for.
template <int kBytes>
__device__ __forceinline__ void copy_piece(uint32_t to, const char* from, bool there) {
  const uint32_t n = there ? kBytes : 0;
  if constexpr (kBytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(kBytes), "r"(n) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void wait_for_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// Where byte `byte` of a row of nibbles or of a token (256 bytes a unit) lies in shared memory.  A row has five pieces
// of 16 bytes: its 64 of a unit may begin within the first.  What a warp reads together lies in different banks: rows are
// 20 words apart, and the halves of a token's 256 bytes change places by the token.
constexpr int kRowPitch = 80;
__device__ __forceinline__ uint32_t row_place(int row, int byte) { return row * kRowPitch + byte; }
__device__ __forceinline__ uint32_t token_place(int token, int byte) { return token * 256 + (byte ^ ((token & 1) << 6)); }

// 16 bytes of a row, but for those outside the whole array, where it ends within them (word by word then).
__device__ __forceinline__ void copy_inside(uint32_t to, const char* from, const Int4Params& p) {
  if (from >= p.w && from + 16 <= p.w_end) {
    copy_piece<16>(to, from, true);
  } else {
#pragma unroll 1
    for (int i = 0; i < 16; i += 4)
      if (from + i >= p.w && from + i < p.w_end) copy_piece<4>(to + i, from + i, true);
  }
}

// The rows of nibbles that a warp copies a unit of: 8 kEach neighbouring ones.
template <int kEach>
struct RowCopies {
  const char* rows[kEach];  // of this lane's rows, from the multiple of 16 bytes that it begins behind
  const char* tail;         // of row `lane`: a fifth piece
  bool first, last;         // whether their first or last pieces may reach out of the array
  static __device__ __forceinline__ const char* aligned(const char* q) {
    return reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(q) & ~uintptr_t(15));
  }
  __device__ __forceinline__ void aim(const Int4Params& p, int64_t row0, int lane) {
    const int64_t end = p.N - 1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) rows[i] = aligned(p.w + min(row0 + i * 8 + (lane >> 2), end) * p.w_rs) + (lane & 3) * 16;
    tail = aligned(p.w + min(row0 + lane, end) * p.w_rs) + 64;
    // (rows may be shorter than a unit, or all the same one: the last tile's are not the only ones)
    first = aligned(p.w + min(row0, end) * p.w_rs) < p.w;
    last = p.w + min(row0 + 8 * kEach - 1, end) * p.w_rs + int64_t(p.units) * 64 + 16 > p.w_end;
  }
  __device__ __forceinline__ void copy(const Int4Params& p, uint32_t to, int lane, int unit) const {
    const uint32_t at = uint32_t(unit) * 64;
    if ((first && unit == 0) || (last && unit >= p.units - 2)) {
#pragma unroll 1
      for (int i = 0; i < kEach; ++i) copy_inside(to + row_place(i * 8 + (lane >> 2), (lane & 3) * 16), rows[i] + at, p);
      if (p.shifted && lane < 8 * kEach) copy_inside(to + row_place(lane, 64), tail + at, p);
      return;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) copy_piece<16>(to + row_place(i * 8 + (lane >> 2), (lane & 3) * 16), rows[i] + at, true);
    if (p.shifted && lane < 8 * kEach) copy_piece<16>(to + row_place(lane, 64), tail + at, true);
  }
};

// The scales (and zero points) of a unit of kGroups groups and of kRows rows, g + 8 r, that four lanes share: value j is of
// group j / kRows and row j % kRows; lane q of the four has those with j % 4 = q, and gives them to the others.
template <int kGroups, int kRows>
struct Scales {
  static constexpr int kOwn = (kRows * kGroups + 3) / 4;
  uint32_t raw[kOwn], zero[kOwn];  // as they come
};
template <int kGroups, int kRows>
struct ScaleRows {
  using Own = Scales<kGroups, kRows>;
  const char* at[Own::kOwn];
  const uint8_t* zero_at[Own::kOwn];
  __device__ __forceinline__ void aim(const Int4Params& p, int64_t row0, int lane) {  // row0: of g = 0
    const int es = p.scale_dtype == CCONV_TYPE_FP32 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < Own::kOwn; ++i) {
      const int64_t r = min(row0 + (lane >> 2) + 8 * ((4 * i + (lane & 3)) % kRows), p.N - 1);
      at[i] = p.scale + r * p.s_rs * es;
      zero_at[i] = p.zero + r * p.z_rs;
    }
  }
  __device__ __forceinline__ void load(const Int4Params& p, int lane, int unit, Own& s) const {
#pragma unroll
    for (int i = 0; i < Own::kOwn; ++i) {
      const int64_t group = unit * kGroups + (4 * i + (lane & 3)) / kRows;
      s.raw[i] = s.zero[i] = 0;  // (behind the last group: nothing times nothing)
      if (group < p.groups && (kRows * kGroups >= 4 || (lane & 3) < kRows * kGroups)) {
        s.raw[i] = load_scale(at[i], p.scale_dtype, group * p.s_cs);
        if (p.zero) s.zero[i] = __ldg(zero_at[i] + group * p.z_cs);
      }
    }
  }
};
// The current unit's.
template <int kGroups, int kRows>
struct ScaleValues {
  using Own = Scales<kGroups, kRows>;
  float by[Own::kOwn];       // scale
  uint32_t low[Own::kOwn];  // zero point
  __device__ __forceinline__ ScaleValues(const Int4Params& p, const Own& s) {
#pragma unroll
    for (int i = 0; i < Own::kOwn; ++i) {
      by[i] = scale_of(s.raw[i], p.scale_dtype);
      low[i] = s.zero[i] & 15u;
    }
  }
  __device__ __forceinline__ float scale(int group, int r, int lane) const {
    const int j = group * kRows + r;
    return __shfl_sync(0xffffffffu, by[j / 4], (lane & 28) | (j & 3));
  }
  __device__ __forceinline__ uint32_t zero_point(const Int4Params& p, int group, int r, int lane) const {
    const int j = group * kRows + r;
    return p.zero ? __shfl_sync(0xffffffffu, low[j / 4], (lane & 28) | (j & 3)) : 8u;
  }
};

// One or two tokens, and up to 8 of small matrices: all of them lie in shared memory, in the order in which the matrix instructions take them, with the
// sums of each group beside them; weights go straight into the registers that multiply them.  A block takes tiles of 16
// kMt rows, blockIdx.x and every gridDim.x-th after it; its warps share k in units of 128, of which a batch is on its way
// while the one before is multiplied, also across tiles.  Of a unit, lane q of the four that share a row takes the
// words of kWords neighbours: no more k than a group has between the four.
template <typename T, int kWords, int kGroups, int kMt>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_int4_kernel(const Int4Params p) {
  // rows of a lane; loads of a unit; units of a batch (32 words a lane, or 16 where scales take registers too)
  constexpr int kRows = 2 * kMt, kSteps = 4 / kWords, kUnits = (kGroups == 1 ? 4 : 2) / kMt;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float sums[kMt * kWarps][128];
  uint4* const tokens = reinterpret_cast<uint4*>(smem);  // [unit][word][token][lane of four]
  float* const totals = reinterpret_cast<float*>(smem + p.units * p.M * 256);  // [unit][group][token]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int tiles = int((p.N + 16 * kMt - 1) / (16 * kMt));
  const int u0 = warp * p.per, u1 = min(p.units, u0 + p.per), batches = (p.per + kUnits - 1) / kUnits;
  const int mine = int(blockIdx.x) < tiles ? (tiles - 1 - int(blockIdx.x)) / int(gridDim.x) + 1 : 0;

  struct Batch {
    Words<kWords> w[kUnits][kSteps][kRows];
    Scales<kGroups, kRows> scales[kUnits];
  } b[2];
  const char* rows[kRows];
  ScaleRows<kGroups, kRows> scale_rows;
  int lt = blockIdx.x, lb = 0;
  auto load = [&](Batch& a) {
    if (lt < tiles) {
      if (lb == 0) {
        const int64_t row0 = int64_t(lt) * (16 * kMt);
        rows[0] = p.w + min(row0 + g, p.N - 1) * p.w_rs + q * (4 * kWords);
#pragma unroll
        for (int r = 1; r < kRows; ++r)
          rows[r] = row0 + 16 * kMt <= p.N ? rows[r - 1] + 8 * p.w_rs : p.w + min(row0 + g + 8 * r, p.N - 1) * p.w_rs + q * (4 * kWords);
        scale_rows.aim(p, row0, lane);
      }
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const int unit = u0 + lb * kUnits + u;
        const uint32_t at = uint32_t(unit) * 64;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const bool in = unit < u1 && at + (i * 4 + q) * (4 * kWords) < p.w_bytes;
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            if (in) a.w[u][i][r].load(rows[r] + at + i * 16 * kWords);
            else a.w[u][i][r].zero();
          }
        }
        if (unit < u1) scale_rows.load(p, lane, unit, a.scales[u]);
      }
    }
    if (++lb == batches) lb = 0, lt += gridDim.x;
  };

  start_in_order();
  load(b[0]);
  {
    // The tokens: eight neighbours of k a thread, four times at once (each alone would wait for memory); the lanes that
    // have a group's add up their sums.
    const int pieces = p.units * 16, all = pieces * p.M;  // (pieces: a multiple of 16, whole groups)
    const unsigned half = (threadIdx.x & 16) ? 0xffff0000u : 0xffffu;
    for (int c0 = threadIdx.x; c0 < all; c0 += 4 * kWarps * 32) {
      uint4 v[4];
      int at[4];  // piece | token << 28
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = c0 + i * kWarps * 32, t = c / pieces, piece = c - t * pieces;
        at[i] = piece | t << 28;
        v[i] = make_uint4(0, 0, 0, 0);
        if (c < all && uint32_t(piece) * 16 < p.x_bytes) v[i] = *reinterpret_cast<const uint4*>(p.x + t * p.x_rs + uint32_t(piece) * 16);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (c0 + i * kWarps * 32 >= all) break;  // (16 threads together)
        const int t = at[i] >> 28, unit = (at[i] & 0xfffffff) >> 4, in = at[i] & 15;
        const int word = in / (4 * kWords) * kWords + in % kWords, four = in / kWords & 3;
        tokens[((unit * 4 + word) * p.M + t) * 4 + four] =
            make_uint4(__byte_perm(v[i].x, v[i].z, 0x5410), __byte_perm(v[i].x, v[i].z, 0x7632), __byte_perm(v[i].y, v[i].w, 0x5410),
                       __byte_perm(v[i].y, v[i].w, 0x7632));
        const float2 f0 = unpack2<T>(v[i].x), f1 = unpack2<T>(v[i].y), f2 = unpack2<T>(v[i].z), f3 = unpack2<T>(v[i].w);
        float sum = ((f0.x + f0.y) + (f1.x + f1.y)) + ((f2.x + f2.y) + (f3.x + f3.y));
#pragma unroll
        for (int o = 1; o < 16 / kGroups; o <<= 1) sum += __shfl_xor_sync(half, sum, o);
        if (in % (16 / kGroups) == 0) totals[(unit * kGroups + in / (16 / kGroups)) * p.M + t] = sum;
      }
    }
  }
  __syncthreads();

  float acc[kMt][4] = {};
  const int token = min(g, p.M - 1), t0 = min(2 * q, p.M - 1), t1 = min(2 * q + 1, p.M - 1);  // (columns behind the last go nowhere)
  int tile = blockIdx.x, batch = 0;
  auto use = [&](Batch& a) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int unit = u0 + batch * kUnits + u;
      if (unit < u1) {
        const ScaleValues<kGroups, kRows> values(p, a.scales[u]);
        float d[kMt][4] = {};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 x = tokens[((unit * 4 + j) * p.M + token) * 4 + q];
#pragma unroll
          for (int m = 0; m < kMt; ++m) {
            const uint32_t lo = a.w[u][j / kWords][2 * m].w[j % kWords], hi = a.w[u][j / kWords][2 * m + 1].w[j % kWords];
            mma16<T>(d[m], two_of<T, 0>(lo, p.base), two_of<T, 0>(hi, p.base), two_of<T, 1>(lo, p.base), two_of<T, 1>(hi, p.base), x.x, x.y);
            mma16<T>(d[m], two_of<T, 2>(lo, p.base), two_of<T, 2>(hi, p.base), two_of<T, 3>(lo, p.base), two_of<T, 3>(hi, p.base), x.z, x.w);
          }
          if ((j + 1) % (4 / kGroups) == 0) {  // a group's sums are complete: scaled and added up
            const int group = j * kGroups / 4;
            const float s0 = totals[(unit * kGroups + group) * p.M + t0], s1 = totals[(unit * kGroups + group) * p.M + t1];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
              const float by = values.scale(group, r, lane), zp = 16.0f + float(values.zero_point(p, group, r, lane));
              float& f0 = d[r >> 1][(r & 1) * 2];
              float& f1 = d[r >> 1][(r & 1) * 2 + 1];
              acc[r >> 1][(r & 1) * 2] += by * (f0 - zp * s0);
              acc[r >> 1][(r & 1) * 2 + 1] += by * (f1 - zp * s1);
              f0 = f1 = 0.0f;
            }
          }
        }
      }
    }
    if (++batch < batches) return;
    batch = 0;
    __syncthreads();  // the tile before has been read
#pragma unroll
    for (int m = 0; m < kMt; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sums[m * kWarps + warp][i * 32 + lane] = acc[m][i];
        acc[m][i] = 0.0f;
      }
    __syncthreads();
    const int64_t n0 = int64_t(tile) * (16 * kMt);
    if (int(threadIdx.x) < 16 * kMt * p.M) {
      // (neighbouring threads: neighbouring rows)
      const int r = threadIdx.x % (16 * kMt), t = threadIdx.x / (16 * kMt), rr = r & 15;
      const float(*part)[128] = sums + (r >> 4) * kWarps;
      const int at = ((rr >> 3) * 2 + (t & 1)) * 32 + (rr & 7) * 4 + (t >> 1);
      float f = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) f += part[w][at];
      if (n0 + r < p.N) static_cast<T*>(const_cast<void*>(p.out.p))[t * p.out.rs + (n0 + r) * p.out.cs] = from_f32<T>(f);
    }
    tile += gridDim.x;
  };
  const int total = mine * batches;
  for (int it = 0; it < total; it += 2) {
    load(b[1]);
    use(b[0]);
    if (it + 1 < total) {
      load(b[0]);
      use(b[1]);
    }
  }
}

constexpr int kStages = 3;

// q - z as pairs of 16-bit numbers, of neighbouring nibbles: bytes that hold a nibble each become the lower bytes of
// 128 + q (bf16) or 1024 + q (fp16), from which 128 + z or 1024 + z (`bias`) is taken off, exactly.
template <typename T>
struct High {
  static constexpr uint32_t kByte = 0x43434343u, kBase = 0x43004300u;
};
template <>
struct High<__half> {
  static constexpr uint32_t kByte = 0x64646464u, kBase = 0x64006400u;
};
template <typename T>
__device__ __forceinline__ uint32_t minus2(uint32_t a, uint32_t b);
template <>
__device__ __forceinline__ uint32_t minus2<__nv_bfloat16>(uint32_t a, uint32_t b) {
  const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t minus2<__half>(uint32_t a, uint32_t b) {
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ void pairs_of(uint32_t v, uint32_t bias, uint32_t (&w)[4]) {
  const uint32_t even = v & 0x0f0f0f0fu, odd = v >> 4 & 0x0f0f0f0fu;
  const uint32_t lo = __byte_perm(even, odd, 0x5140), hi = __byte_perm(even, odd, 0x7362);
  w[0] = minus2<T>(__byte_perm(lo, High<T>::kByte, 0x4140), bias);
  w[1] = minus2<T>(__byte_perm(lo, High<T>::kByte, 0x4342), bias);
  w[2] = minus2<T>(__byte_perm(hi, High<T>::kByte, 0x4140), bias);
  w[3] = minus2<T>(__byte_perm(hi, High<T>::kByte, 0x4342), bias);
}

// Up to 64 tokens: their words, not the weights, would fill the shared memory's bandwidth if each warp fetched its own.  So
// the warps of a block share the tokens of a unit and take 16 rows each; a cluster of `parts` blocks shares k, and
// adds up its sums through distributed shared memory in a fixed order.
template <int kNt>
constexpr int kSharedUnit = 16 * kWarps * kRowPitch + 8 * kNt * 256;
template <typename T, int kGroups, int kNt>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_int4_tokens_kernel(const Int4Params p, const int parts) {
  constexpr int kUnitBytes = kSharedUnit<kNt>, kWeightBytes = 16 * kWarps * kRowPitch;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int rank = int(blockIdx.x) % parts;
  const int64_t n0 = int64_t(blockIdx.x) / parts * (16 * kWarps), row0 = n0 + warp * 16;
  const int u0 = int(int64_t(p.units) * rank / parts), u1 = int(int64_t(p.units) * (rank + 1) / parts);
  const int token = int(threadIdx.x >> 4);
  const char* const token_from = p.x + token * p.x_rs;
  const uint32_t token_at = smem_u32(smem) + kWeightBytes + token_place(token, (lane & 15) * 16);
  RowCopies<2> rows;
  rows.aim(p, row0, lane);
  ScaleRows<kGroups, 2> scale_rows;
  scale_rows.aim(p, row0, lane);
  Scales<kGroups, 2> scales;
  auto load = [&](int stage, int unit) {
    if (unit < u1) {
      rows.copy(p, smem_u32(smem) + stage * kUnitBytes + warp * (16 * kRowPitch), lane, unit);
      const uint32_t at = uint32_t(unit) * 256 + (lane & 15) * 16;
      const bool there = at < p.x_bytes;
#pragma unroll
      for (int i = 0; i < (kNt + 1) / 2; ++i)
        if (i * 16 + token < p.M) copy_piece<16>(token_at + stage * kUnitBytes + i * 4096, token_from + i * 16 * p.x_rs + (there ? at : 0), there);
    }
    commit_copies();
  };

  start_in_order();
  for (int i = 0; i < kStages - 1; ++i) load(i, u0 + i);
  if (u0 < u1) scale_rows.load(p, lane, u0, scales);
  uint32_t word[2];
#pragma unroll
  for (int r = 0; r < 2; ++r)
    word[r] = row_place(warp * 16 + g + 8 * r,
                        int((reinterpret_cast<uintptr_t>(p.w) + uint64_t(min(row0 + g + 8 * r, p.N - 1) * p.w_rs)) & 15) + q * 4);
  const uint32_t x_word[2] = {kWeightBytes + token_place(g, q * 16), kWeightBytes + token_place(g, 64 + q * 16)};
  float acc[kNt][4] = {};
  int stage = 0;
  for (int unit = u0; unit < u1; ++unit) {
    const ScaleValues<kGroups, 2> values(p, scales);
    if (unit + 1 < u1) scale_rows.load(p, lane, unit + 1, scales);
    wait_for_copies<kStages - 2>();
    __syncthreads();  // the unit is there for all, and the one before has been read by all
    load(stage == 0 ? kStages - 1 : stage - 1, unit + kStages - 1);
    const uint8_t* const from = smem + stage * kUnitBytes;
    if (++stage == kStages) stage = 0;
    float d[kNt][4] = {};
    uint32_t bias[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i % (4 / kGroups) == 0) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
          bias[r] = High<T>::kBase | values.zero_point(p, i * kGroups / 4, r, lane) * 0x10001u;
      }
      uint32_t lo[4], hi[4];
      pairs_of<T>(*reinterpret_cast<const uint32_t*>(from + word[0] + i * 16), bias[0], lo);
      pairs_of<T>(*reinterpret_cast<const uint32_t*>(from + word[1] + i * 16), bias[1], hi);
#pragma unroll
      for (int e = 0; e < kNt; ++e) {
        // (columns behind the last token: whatever lies there, for sums that go nowhere)
        const uint4 v = *reinterpret_cast<const uint4*>(from + x_word[i & 1] + (i >> 1) * 128 + e * 2048);
        mma16<T>(d[e], lo[0], hi[0], lo[1], hi[1], v.x, v.y);
        mma16<T>(d[e], lo[2], hi[2], lo[3], hi[3], v.z, v.w);
      }
      if ((i + 1) % (4 / kGroups) == 0) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float by = values.scale(i * kGroups / 4, r, lane);
#pragma unroll
          for (int e = 0; e < kNt; ++e)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              acc[e][r * 2 + c] += by * d[e][r * 2 + c];
              d[e][r * 2 + c] = 0.0f;
            }
        }
      }
    }
  }
  __syncthreads();
  // sums as [token][row] in the ring's place
  float* const sums = reinterpret_cast<float*>(smem);
  constexpr int kPitch = 16 * kWarps + 4;
#pragma unroll
  for (int e = 0; e < kNt; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 8 * e + 2 * q + (i & 1);
      if (t < p.M) sums[t * kPitch + warp * 16 + g + (i >> 1) * 8] = acc[e][i];
    }
  if (parts > 1) cluster_sync_all();
  else __syncthreads();
  for (int i = threadIdx.x + rank * kWarps * 32; i < p.M * 16 * kWarps; i += parts * kWarps * 32) {
    const int r = i % (16 * kWarps), t = i / (16 * kWarps);
    float f = 0.0f;
    if (parts > 1) {
      const uint32_t at = smem_u32(sums + t * kPitch + r);
      for (int b = 0; b < parts; ++b) f += load_cluster(cluster_map_shared(at, b));
    } else {
      f = sums[t * kPitch + r];
    }
    if (n0 + r < p.N) static_cast<T*>(const_cast<void*>(p.out.p))[t * p.out.rs + (n0 + r) * p.out.cs] = from_f32<T>(f);
  }
  if (parts > 1) cluster_sync_all();  // no block leaves while others read its sums
}

// The weights as numbers of the operands' type, for products of many tokens: 8 or 16 neighbours of a row a thread, 4 rows.
// Bound by the store of 2 bytes a weight, where scales are of that type too (one rounding, of an exact product, a pair).
// The rounding is to the operands' precision: the tensor cores take nothing finer of that type.  Its range is bf16's, which
// is the scales' own; in fp16 weights would leave it from scales of 4367 on and lose bits below 6e-5, so that there a row
// is divided by a power of two that brings its largest scale to [2^10, 2^11) (times 15: below 2^15), and the product's
// columns are multiplied by it in fp32.  What a row's small groups lose to fp16's smallest step is 2^-31 of its largest scale.
struct ExpandParams {
  const char *w, *scale;
  const uint8_t* zero;
  void* to;
  int64_t w_rs, s_rs, s_cs, z_rs, z_cs, to_rs, N, K;
  float* power;  // [N], written: of fp16 weights
  int groups;
  int scale_dtype, group_shift;  // 1 << group_shift words a group
};
template <typename T>
__device__ __forceinline__ uint32_t times2(uint32_t a, uint32_t b);
template <>
__device__ __forceinline__ uint32_t times2<__nv_bfloat16>(uint32_t a, uint32_t b) {
  const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t times2<__half>(uint32_t a, uint32_t b) {
  const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
constexpr int kExpandRows = 4;
// A row's power of two, by a warp.  Scales that are not finite are not looked at: their weights stay so.  (From 2^-100 on
// both it and its inverse are normal numbers; smaller scales give results that round to 0.)
__device__ __forceinline__ float power_of_row(const char* scale, int scale_dtype, int64_t s_cs, int groups) {
  uint32_t most = 0;
  for (int i = threadIdx.x & 31; i < groups; i += 32) {
    const uint32_t size = __float_as_uint(scale_of(load_scale(scale, scale_dtype, i * s_cs), scale_dtype)) & 0x7fffffffu;
    if (size < 0x7f800000u) most = max(most, size);
  }
  most = __reduce_max_sync(0xffffffffu, most);
  const int e = most ? max(ilogbf(__uint_as_float(most)) - 10, -100) : 0;
  return __uint_as_float(uint32_t(127 + e) << 23);
}
__device__ __forceinline__ float inverse_of_power(float v) { return __uint_as_float((254u << 23) - __float_as_uint(v)); }
// kWords neighbouring words a thread (2 where that keeps to multiples of 32 bytes, which go in one store); kSame: scales
// are of the type T.
template <typename T, int kWords, bool kSame>
__global__ void __launch_bounds__(256, 4) cconv_int4_expand_kernel(const ExpandParams p) {
  constexpr bool kPowers = std::is_same<T, __half>::value;
  __shared__ float inverse[2][kExpandRows];
  start_in_order();
  const uint32_t words = uint32_t((p.K + 7) / 8), i = (blockIdx.x * 256 + threadIdx.x) * kWords;
  const bool inside = i < words;
  if (!kPowers && !inside) return;
  int turn = 0;
  const int64_t grp = i >> p.group_shift;
  const int es = kSame || p.scale_dtype != CCONV_TYPE_FP32 ? 2 : 4;
  const int64_t scale_step = p.s_rs * es, to_step = p.to_rs * int64_t(sizeof(T));
  for (int64_t n0 = int64_t(blockIdx.y) * kExpandRows; n0 < p.N; n0 += int64_t(gridDim.y) * kExpandRows) {
    const int rows = int(min(p.N - n0, int64_t(kExpandRows)));
    const char* w_at = p.w + n0 * p.w_rs + i * 4;
    const char* s_at = p.scale + (n0 * p.s_rs + grp * p.s_cs) * es;
    const uint8_t* z_at = p.zero + n0 * p.z_rs + grp * p.z_cs;
    char* to = static_cast<char*>(p.to) + n0 * to_step + i * 16;
    Words<kWords> v[kExpandRows];
    uint32_t s[kExpandRows], z[kExpandRows];
#pragma unroll
    for (int r = 0; r < kExpandRows; ++r, w_at += p.w_rs, s_at += scale_step, z_at += p.z_rs) {
      z[r] = 8;
      if (r >= rows || !inside) break;
      v[r].load(w_at);
      if (es == 2) s[r] = __ldg(reinterpret_cast<const uint16_t*>(s_at));
      else s[r] = __ldg(reinterpret_cast<const uint32_t*>(s_at));
      if (p.zero) z[r] = __ldg(z_at) & 15u;
    }
    if constexpr (kPowers) {
      const int warp = threadIdx.x >> 5;
      if (warp < rows) {  // (warps 0 to 3)
        const float power = power_of_row(p.scale + (n0 + warp) * scale_step, p.scale_dtype, p.s_cs, p.groups);
        if ((threadIdx.x & 31) == 0) {
          inverse[turn][warp] = inverse_of_power(power);
          if (blockIdx.x == 0) p.power[n0 + warp] = power;
        }
      }
      __syncthreads();  // (the next rows' go to the other half, which all have read by the barrier after)
    }
#pragma unroll
    for (int r = 0; r < kExpandRows; ++r, to += to_step) {
      if (r >= rows || !inside) break;
      const float times = kPowers ? inverse[turn][r] : 1.0f;
      if (kPowers && kSame) s[r] = __half_as_ushort(__float2half_rn(scale_of(s[r], CCONV_TYPE_FP16) * times));
      uint32_t w[kWords][4];
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        pairs_of<T>(v[r].w[k], High<T>::kBase | z[r] * 0x10001u, w[k]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (kSame) {
            w[k][j] = times2<T>(w[k][j], s[r] * 0x10001u);
          } else {
            const float by = scale_of(s[r], p.scale_dtype) * times;
            const float2 f = unpack2<T>(w[k][j]);
            w[k][j] = pack2<T>(by * f.x, by * f.y);
          }
        }
      }
      if constexpr (kWords == 2) st_global_v8(to, w[0][0], w[0][1], w[0][2], w[0][3], w[1][0], w[1][1], w[1][2], w[1][3]);
      else *reinterpret_cast<uint4*>(to) = make_uint4(w[0][0], w[0][1], w[0][2], w[0][3]);
    }
    turn ^= 1;
  }
}

constexpr int kMostTokenBytes = 96 * 1024;  // of shared memory, so that two blocks share an SM

template <typename T, int kWords, int kGroups, int kMt>
cudaError_t launch_rows(const Int4Params& p, int sms, cudaStream_t s) {
  auto f = cconv_int4_kernel<T, kWords, kGroups, kMt>;
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, kSpreadSmem);
  if (e != cudaSuccess) return e;
  const dim3 grid(unsigned(std::min<int64_t>(cdiv64(p.N, 16 * kMt), 2 * sms)));
  return launch(f, grid, kWarps * 32, size_t(spread_smem(grid.x, sms, p.units * p.M * (256 + kGroups * 4))), 1, s, p);
}
template <typename T, int kGroups, int kNt>
cudaError_t launch_shared(const Int4Params& p, int sms, cudaStream_t s) {
  auto f = cconv_int4_tokens_kernel<T, kGroups, kNt>;
  constexpr int kSmem = std::max(kStages * kSharedUnit<kNt>, 8 * kNt * (16 * kWarps + 4) * 4);
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, std::max(kSmem, kSpreadSmem));
  if (e != cudaSuccess) return e;
  const int64_t tiles = cdiv64(p.N, 16 * kWarps);
  // As many parts as leave every block its place at once, two an SM.  A cluster lies in one group of SMs, whose number
  // differs, so that the device is asked: 40 tiles (5000 x 4200, 23 tokens) in 4 parts 16.5 us, in 6 13.2, in 7, which do
  // not fit, 20.  (Not quite all places, while the kernel in front may still have some: 55 tiles in 5 parts 14 us, in 4 12.5.)
  static std::atomic<int> places[64][9];
  int parts = 1;
  for (int n = 2; n <= 8 && n <= p.units && tiles * n <= 2 * sms - sms / 4; ++n) {
    int at_once = 0;
    const cudaError_t e = clusters_at_once(f, kWarps * 32, std::max(kSmem, spread_smem(2, 1, 0)), n, places, &at_once);
    if (e != cudaSuccess) return e;
    if (tiles <= at_once) parts = n;
  }
  const int64_t blocks = tiles * parts, apart = parts > 1 ? std::max<int64_t>(blocks, sms + 1) : blocks;
  return launch(f, dim3(unsigned(blocks)), kWarps * 32, size_t(spread_smem(apart, sms, kSmem)), parts, s, p, parts);
}
template <typename T, int kWords, int kGroups>
cudaError_t launch_words(const Int4Params& p, int sms, cudaStream_t s) {
  // 32 rows a tile where that leaves no SM idle
  return cdiv64(p.N, 32) >= sms ? launch_rows<T, kWords, kGroups, 2>(p, sms, s) : launch_rows<T, kWords, kGroups, 1>(p, sms, s);
}
template <typename T, int kGroups>
cudaError_t launch_tokens(const Int4Params& p, int sms, cudaStream_t s) {
  if (p.M > 48) return launch_shared<T, kGroups, 8>(p, sms, s);
  if (p.M > 32) return launch_shared<T, kGroups, 6>(p, sms, s);
  if (p.M > 24) return launch_shared<T, kGroups, 4>(p, sms, s);
  if (p.M > 16) return launch_shared<T, kGroups, 3>(p, sms, s);
  if (p.M > 8) return launch_shared<T, kGroups, 2>(p, sms, s);
  // What each block makes of the tokens for itself takes longer than its tile's weights once they are several, but for
  // small matrices: 8 tokens 4096 x 4096 8.4 against 6.7 us shared, 2048 x 2048 4.8 against 5.6.
  const bool own = p.M <= 2 || p.units * p.M <= 128;
  if (!own || int64_t(p.units) * p.M * (256 + kGroups * 4) > kMostTokenBytes) return launch_shared<T, kGroups, 1>(p, sms, s);
  constexpr int kWords = 4 / kGroups;  // that four lanes may have of a group
  const int most = (p.lies & 15) == 0 ? 4 : (p.lies & 7) == 0 ? 2 : 1;
  if constexpr (kWords == 4)
    if (most == 4) return launch_words<T, 4, kGroups>(p, sms, s);
  if constexpr (kWords >= 2)
    if (most >= 2) return launch_words<T, 2, kGroups>(p, sms, s);
  return launch_words<T, 1, kGroups>(p, sms, s);
}
template <typename T>
cudaError_t launch_few(const Int4Params& p, int group, int sms, cudaStream_t s) {
  if (group == 128) return launch_tokens<T, 1>(p, sms, s);
  if (group == 64) return launch_tokens<T, 2>(p, sms, s);
  return launch_tokens<T, 4>(p, sms, s);
}

constexpr int64_t kFewTokensInt4 = 64;

void plan(Steps& st, const cconv_int4_product_args& a) {
  const int64_t M = a.M, N = a.N, K = a.K, row = cdiv64(K, 2);
  const int dtype = a.dtype, sms = st.sms(), group = a.group;
  // Rows of nibbles that words can be read from, in place or copied.
  Mat w(a.q);
  int64_t w_bytes = row;
  uintptr_t at = reinterpret_cast<uintptr_t>(a.q.data) | uintptr_t(N > 1 ? a.q.row_stride : 0);
  if (K % 8 || (at & 3) || (a.q.col_stride != 1 && row > 1)) {
    w = st.scratch(N, row, 1);
    w_bytes = w.rs;
    at = 0;
    st.copy(Mat(a.q), w, N, row, 1);
  }
  if (M <= kFewTokensInt4) {
    Int4Params p{};
    int64_t readable = 0;
    Padded padded;
    const Mat x = padded.readable(st, a.x, M, K, &readable);
    padded.add(st);
    p.x_bytes = uint32_t(readable) * 2;
    p.x = static_cast<const char*>(x.p);
    p.x_rs = x.rs * 2;
    p.w = static_cast<const char*>(w.p);
    p.w_rs = w.rs;
    p.w_end = p.w + (N - 1) * w.rs + w_bytes;
    p.shifted = (at & 15) != 0;
    p.w_bytes = uint32_t(w_bytes);
    p.lies = uint32_t((at | uintptr_t(w_bytes)) & 15);
    p.scale = static_cast<const char*>(a.scale.data);
    p.s_rs = a.scale.row_stride; p.s_cs = a.scale.col_stride;
    p.zero = static_cast<const uint8_t*>(a.zero.data);
    p.z_rs = a.zero.row_stride; p.z_cs = a.zero.col_stride;
    p.N = N;
    p.M = int(M);
    p.scale_dtype = a.scale_dtype;
    p.groups = int(cdiv64(K, group));
    p.units = int(cdiv64(K, 128));
    p.per = int(cdiv64(p.units, kWarps));
    p.out = Mat(a.c);
    p.base = dtype == CCONV_TYPE_BF16 ? Code<__nv_bfloat16>::kBase : Code<__half>::kBase;
    st.add([=](cudaStream_t s) {
      return block_cuda_error(dtype == CCONV_TYPE_BF16 ? launch_few<__nv_bfloat16>(p, group, sms, s)
                                                       : launch_few<__half>(p, group, sms, s),
                              "cconv_int4_kernel");
    });
    return;
  }
  ExpandParams p{};
  const Mat full = st.scratch(N, K, 2);
  p.w = static_cast<const char*>(w.p);
  p.w_rs = w.rs;
  p.scale = static_cast<const char*>(a.scale.data);
  p.s_rs = a.scale.row_stride; p.s_cs = a.scale.col_stride;
  p.zero = static_cast<const uint8_t*>(a.zero.data);
  p.z_rs = a.zero.row_stride; p.z_cs = a.zero.col_stride;
  p.to = const_cast<void*>(full.p);
  p.to_rs = full.rs;
  p.N = N;
  p.K = K;
  p.scale_dtype = a.scale_dtype;
  p.groups = int(cdiv64(K, group));
  p.group_shift = group == 32 ? 2 : group == 64 ? 3 : 4;
  const bool two = K % 16 == 0 && (at & 7) == 0;
  Mat powers;
  if (dtype == CCONV_TYPE_FP16) {
    powers = st.scratch(1, round_up64(N, 256), 4);
    p.power = static_cast<float*>(const_cast<void*>(powers.p));
  }
  st.add([=](cudaStream_t s) {
    const dim3 grid(unsigned(cdiv64(K, two ? 4096 : 2048)), unsigned(std::min<int64_t>(cdiv64(N, kExpandRows), 65535)));
    auto go = [&](auto f) { return block_cuda_error(launch(f, grid, 256, 0, 1, s, p), "cconv_int4_expand_kernel"); };
    auto of = [&](auto type) {
      using T = decltype(type);
      if (p.scale_dtype == dtype) return two ? go(cconv_int4_expand_kernel<T, 2, true>) : go(cconv_int4_expand_kernel<T, 1, true>);
      return two ? go(cconv_int4_expand_kernel<T, 2, false>) : go(cconv_int4_expand_kernel<T, 1, false>);
    };
    return dtype == CCONV_TYPE_BF16 ? of(__nv_bfloat16()) : of(__half());
  });
  Launch l;
  l.epilogue = dtype == CCONV_TYPE_FP16 ? kColumns : kStore;
  l.col_scale = powers;
  l.dtype = dtype;
  l.of[0].M = M;
  l.of[0].N = N;
  l.of[0].K = K;
  l.of[0].a[0] = st.operand(Mat(a.x), M, K);
  operand_in_place(full, N, K, 2, false, &l.of[0].b[0]);
  choose_cut(&l, sms, true);
  const Mat to[3] = {Mat(a.c), Mat(), Mat()};
  st.launch(l, to);
}

// ---- quantiser ---------------------------------------------------------------------------------
struct GroupParams {
  const void* w;
  int64_t w_rs, w_cs;
  uint8_t* q;
  int64_t q_rs, q_cs;
  void* scale;
  int64_t s_rs, s_cs;
  uint8_t* zero;
  int64_t z_rs, z_cs, N, K;
  int scale_dtype;
};

__device__ __forceinline__ float round_to(float v, int dtype) {
  if (dtype == CCONV_TYPE_BF16) return __bfloat162float(__float2bfloat16_rn(v));
  if (dtype == CCONV_TYPE_FP16) return __half2float(__float2half_rn(v));
  return v;
}

// Eight neighbours of a row a lane, kGroup / 8 lanes a group.  One pass: a group's values stay in registers between
// their extremes and their rounding.
template <typename T, int kGroup>
__global__ void __launch_bounds__(256) cconv_quantize_groups_kernel(const GroupParams p, const bool wide) {
  constexpr int kLanes = kGroup / 8;
  start_in_order();
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x, k0 = i * 8;  // (whole groups; those behind K do nothing)
  for (int64_t n = blockIdx.y; n < p.N; n += gridDim.y) {
    const T* from = static_cast<const T*>(p.w) + n * p.w_rs;
    const int64_t left = p.K - k0;
    float f[8];
    if (wide) {
      union { uint4 v[sizeof(T) / 2]; T t[8]; } in;
#pragma unroll
      for (int j = 0; j < int(sizeof(T) / 2); ++j)
        in.v[j] = left > 0 ? __ldg(reinterpret_cast<const uint4*>(from + k0) + j) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = to_f32(in.t[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = j < left ? to_f32(from[(k0 + j) * p.w_cs]) : 0.0f;
    }
    // zeros change neither extreme, which take in 0
    float lo = 0.0f, hi = 0.0f;
    bool nan = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      lo = fminf(lo, f[j]);
      hi = fmaxf(hi, f[j]);
      nan |= f[j] != f[j];
    }
    if (nan) hi = __int_as_float(0x7f800000), lo = -hi;  // (told from an infinity below: both make a scale that is not finite)
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) {
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const bool finite = hi < __int_as_float(0x7f800000) && lo > -__int_as_float(0x7f800000);
    float s = round_to(p.zero ? __fdiv_rn(hi - lo, 15.0f) : __fdiv_rn(fmaxf(hi, -lo), 7.0f), p.scale_dtype);
    if (!finite) s = __int_as_float(0x7fffffff);
    const bool usable = s > 0.0f && s < __int_as_float(0x7f800000);
    const float z = usable && p.zero ? fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.0f), 15.0f) : 8.0f;
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = usable ? fminf(fmaxf(rintf(__fdiv_rn(f[j], s)) + z, 0.0f), 15.0f) : 8.0f;
      word |= uint32_t(int(v)) << (4 * j);
    }
    if (left <= 0) continue;
    if (left < 8) word &= 0xffffffffu >> (32 - 4 * int(left));  // the nibble behind an odd K is 0
    uint8_t* to = p.q + n * p.q_rs;
    const int64_t at = k0 / 2;
    if (wide) {
      *reinterpret_cast<uint32_t*>(to + at) = word;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (2 * j < left) to[(at + j) * p.q_cs] = uint8_t(word >> (8 * j));
    }
    if (k0 % kGroup == 0) {
      const int64_t grp = k0 / kGroup, as = n * p.s_rs + grp * p.s_cs;
      if (p.scale_dtype == CCONV_TYPE_BF16) static_cast<__nv_bfloat16*>(p.scale)[as] = __float2bfloat16_rn(s);
      else if (p.scale_dtype == CCONV_TYPE_FP16) static_cast<__half*>(p.scale)[as] = __float2half_rn(s);
      else static_cast<float*>(p.scale)[as] = s;
      if (p.zero) p.zero[n * p.z_rs + grp * p.z_cs] = uint8_t(int(z));
    }
  }
}

template <typename T>
cudaError_t launch_groups(const GroupParams& p, int group, cudaStream_t s) {
  const bool wide = p.K % 8 == 0 && p.w_cs == 1 && p.q_cs == 1 &&
                    ((reinterpret_cast<uintptr_t>(p.w) | uintptr_t(p.w_rs * int64_t(sizeof(T)))) & 15) == 0 &&
                    ((reinterpret_cast<uintptr_t>(p.q) | uintptr_t(p.q_rs)) & 3) == 0;
  const dim3 grid(unsigned(cdiv64(p.K, 2048)), unsigned(std::min<int64_t>(p.N, 65535)));
  if (group == 32) return launch(cconv_quantize_groups_kernel<T, 32>, grid, 256, 0, 1, s, p, wide);
  if (group == 64) return launch(cconv_quantize_groups_kernel<T, 64>, grid, 256, 0, 1, s, p, wide);
  return launch(cconv_quantize_groups_kernel<T, 128>, grid, 256, 0, 1, s, p, wide);
}

}  // namespace

int64_t int4_workspace(const cconv_int4_product_args& a, int sms) {
  Steps st(nullptr, sms, 2, a.dtype);
  plan(st, a);
  return st.bytes();
}

int run_int4(const cconv_int4_product_args& a, int sms, cudaStream_t s) {
  Steps st(a.workspace, sms, 2, a.dtype);
  plan(st, a);
  return st.run(s);
}

cudaError_t run_quantize_groups(const cconv_quantize_groups_args& a, cudaStream_t s) {
  GroupParams p{};
  p.w = a.w.data; p.w_rs = a.w.row_stride; p.w_cs = a.w.col_stride;
  p.q = static_cast<uint8_t*>(a.q.data); p.q_rs = a.q.row_stride; p.q_cs = a.q.col_stride;
  p.scale = a.scale.data; p.s_rs = a.scale.row_stride; p.s_cs = a.scale.col_stride;
  p.zero = static_cast<uint8_t*>(a.zero.data); p.z_rs = a.zero.row_stride; p.z_cs = a.zero.col_stride;
  p.N = a.N;
  p.K = a.K;
  p.scale_dtype = a.scale_dtype;
  if (a.dtype == CCONV_TYPE_BF16) return launch_groups<__nv_bfloat16>(p, a.group, s);
  if (a.dtype == CCONV_TYPE_FP16) return launch_groups<__half>(p, a.group, s);
  return launch_groups<float>(p, a.group, s);
}

}  // namespace cconv
