// Products with weights of 4 bits and a scale for each group of 32, 64 or 128 of a row, and their quantiser.
//
//   C[m][n] = sum_g s[n][g] sum_{k in g} (q[n][k] - z[n][g]) x[m][k]
//           = sum_g s[n][g] (sum_k (16 + q) x - (16 + z) sum_k x)
//
// Few tokens: the weights are read once, through shared memory into warp-wide matrix instructions.  16 + q
// is a 16-bit number whose mantissa starts with the four bits, so that a shift and a logical operation make two of
// them; a group's sums come out of the matrix instructions, those of x beside them (rows of ones), and are scaled and
// added up in fp32.  16 + q against q - z costs a factor of 5 in the sums' rounding, 2^-21 in place of 2^-23.
//
// A word holds k = 0 .. 7 in its nibbles; the two that one shift brings in place are four apart, so x's pairs are
// taken four apart too.
#include "block_int4.h"

#include <algorithm>
#include <type_traits>

#include "block_device.cuh"
#include "block_few.h"
#include "block_gemm.h"
#include "block_launch.h"
#include "block_mma.cuh"
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
  static constexpr uint32_t kMask = 0x00780078u, kBase = 0x41804180u, kOnes = 0x3f803f80u;
};
template <>
struct Code<__half> {
  static constexpr int kAt = 6;
  static constexpr uint32_t kMask = 0x03c003c0u, kBase = 0x4c004c00u, kOnes = 0x3c003c00u;
};
// 16 + q of nibbles i and i + 4.
template <typename T, int i>
__device__ __forceinline__ uint32_t two_of(uint32_t v) {
  constexpr int kShift = Code<T>::kAt - 4 * i;
  const uint32_t at = kShift >= 0 ? v << (kShift & 31) : v >> (-kShift & 31);
  return (at & Code<T>::kMask) | Code<T>::kBase;
}

struct Int4Params {
  const char *x, *w;  // tokens by k; rows of nibbles
  int64_t x_rs, w_rs;  // bytes
  const char* scale;
  const uint8_t* zero;
  int64_t s_rs, s_cs, z_rs, z_cs;  // elements
  int64_t N, x_k, w_bytes;  // x_k, w_bytes: of a row that may be read, multiples of 8 elements and of a piece
  int M, scale_dtype, piece, groups;
  int units, per;  // of 128 of k; of a warp
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

// Where byte `byte` of a row of nibbles (64 bytes a unit) or of a token (256 bytes a unit) lies in shared memory: 16-byte
// pieces change places by the row, so that what a warp reads together lies in different banks.
__device__ __forceinline__ uint32_t row_place(int row, int byte) { return row * 64 + (byte ^ ((row >> 1 & 3) << 4)); }
__device__ __forceinline__ uint32_t token_place(int token, int byte) { return token * 256 + (byte ^ ((token & 1) << 6)); }

// Copies a unit of 8 kEach rows of nibbles: row_of(r) is where row r begins.
template <int kEach, typename Row>
__device__ __forceinline__ void copy_rows(uint32_t to, int lane, const Int4Params& p, const char* const (&rows)[kEach], int unit, Row row_of) {
  if (p.piece == 16) {  // (rows: those of this lane)
    const int64_t at = int64_t(unit) * 64 + (lane & 3) * 16;
    const bool there = at < p.w_bytes;
#pragma unroll
    for (int i = 0; i < kEach; ++i) copy_piece<16>(to + row_place(i * 8 + (lane >> 2), (lane & 3) * 16), rows[i] + (there ? at : 0), there);
    return;
  }
  auto pieces = [&](auto bytes) {
    constexpr int kBytes = decltype(bytes)::value, kAcross = 64 / kBytes;
#pragma unroll 4
    for (int c = lane; c < 8 * kEach * kAcross; c += 32) {
      const int r = c / kAcross, off = c % kAcross * kBytes;
      const int64_t at = int64_t(unit) * 64 + off;
      const bool there = at < p.w_bytes;
      copy_piece<kBytes>(to + row_place(r, off), row_of(r) + (there ? at : 0), there);
    }
  };
  if (p.piece == 8) pieces(std::integral_constant<int, 8>());
  else pieces(std::integral_constant<int, 4>());
}

// Up to 8 tokens.  A block takes tiles of 16 kMt rows, blockIdx.x and every gridDim.x-th after it; its warps share k in
// units of 128.  Each warp copies its units, weights and tokens, to a ring of its own in shared memory, also across
// tiles: where a block has a tile or two, nearly all that it reads is on its way at once.  Scales come with the unit into
// registers, a fourth of them to each of the four lanes that share a row.
constexpr int kStages = 3;
template <typename T, int kGroups, int kMt>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_int4_kernel(const Int4Params p) {
  constexpr int kRows = 2 * kMt;  // rows of a lane
  constexpr int kScales = (kRows * kGroups + 3) / 4, kWeightBytes = 16 * kMt * 64;
  extern __shared__ __align__(128) uint8_t smem[];
  float(*const sums)[128] = reinterpret_cast<float(*)[128]>(smem);  // [kMt * kWarps]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int unit_bytes = kWeightBytes + p.M * 256;
  const uint8_t* const ring = smem + kMt * kWarps * 512 + warp * (kStages * unit_bytes);
  const uint32_t ring_at = smem_u32(ring);
  const int tiles = int((p.N + 16 * kMt - 1) / (16 * kMt));
  const int u0 = warp * p.per;
  const int mine = int(blockIdx.x) < tiles ? (tiles - 1 - int(blockIdx.x)) / int(gridDim.x) + 1 : 0;
  const int64_t last = p.N - 1;

  uint32_t scale[kStages][kScales], zero[kStages][kScales];
  int lt = blockIdx.x, lu = 0;
  const char *rows[kRows], *scales[kScales];  // of the tile: what this lane copies of, and its scales' rows
  const uint8_t* zeros[kScales];
  const int scale_bytes = p.scale_dtype == CCONV_TYPE_FP32 ? 4 : 2;
  auto row_of = [&](int r) { return p.w + min(int64_t(lt) * (16 * kMt) + r, last) * p.w_rs; };
  // scale number j of a unit: group j / kRows, row j % kRows; lane q has those with j % 4 = q
  auto aim = [&]() {
#pragma unroll
    for (int i = 0; i < kRows; ++i) rows[i] = row_of(i * 8 + (lane >> 2));
#pragma unroll
    for (int i = 0; i < kScales; ++i) {
      const int64_t r = min(int64_t(lt) * (16 * kMt) + g + 8 * ((4 * i + q) % kRows), last);
      scales[i] = p.scale + r * p.s_rs * scale_bytes;
      zeros[i] = p.zero + r * p.z_rs;
    }
  };
  auto load = [&](int stage, uint32_t (&s)[kScales], uint32_t (&z)[kScales]) {
    const int unit = u0 + lu;
    if (lt < tiles && unit < p.units) {
      const uint32_t to = ring_at + stage * unit_bytes;
      copy_rows(to, lane, p, rows, unit, row_of);
      const int64_t k0 = int64_t(unit) * 128 + (lane & 15) * 8;
      const bool there = k0 < p.x_k;
      for (int t = lane >> 4; t < p.M; t += 2)
        copy_piece<16>(to + kWeightBytes + token_place(t, (lane & 15) * 16), p.x + t * p.x_rs + (there ? k0 * 2 : 0), there);
#pragma unroll
      for (int i = 0; i < kScales; ++i) {
        const int64_t grp = min(unit * kGroups + (4 * i + q) / kRows, p.groups - 1);
        s[i] = load_scale(scales[i], p.scale_dtype, grp * p.s_cs);
        if (p.zero) z[i] = __ldg(zeros[i] + grp * p.z_cs);
      }
    }
    commit_copies();
    if (++lu == p.per) {
      lu = 0;
      lt += gridDim.x;
      aim();
    }
  };

  start_in_order();
  aim();
#pragma unroll
  for (int i = 0; i < kStages; ++i) load(i, scale[i], zero[i]);

  float acc[kMt][4] = {};
  int tile = blockIdx.x, step = 0;
  auto use = [&](int stage, const uint32_t (&s)[kScales], const uint32_t (&z)[kScales]) {
    const int unit = u0 + step;
    wait_for_copies<kStages - 1>();
    __syncwarp();
    if (unit < p.units) {
      const uint8_t* const from = ring + stage * unit_bytes;
      float d[kMt][4] = {}, sum[4] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) w[r] = *reinterpret_cast<const uint32_t*>(from + row_place(g + 8 * r, i * 16 + q * 4));
        // (a column behind the last token repeats it and goes nowhere)
        const uint4 v = *reinterpret_cast<const uint4*>(from + kWeightBytes + token_place(min(g, p.M - 1), i * 64 + q * 16));
        const uint32_t x0 = __byte_perm(v.x, v.z, 0x5410), x1 = __byte_perm(v.x, v.z, 0x7632);
        const uint32_t x2 = __byte_perm(v.y, v.w, 0x5410), x3 = __byte_perm(v.y, v.w, 0x7632);
        constexpr uint32_t one = Code<T>::kOnes;
        mma16<T>(sum, one, one, one, one, x0, x1);
        mma16<T>(sum, one, one, one, one, x2, x3);
#pragma unroll
        for (int m = 0; m < kMt; ++m) {
          const uint32_t lo = w[2 * m], hi = w[2 * m + 1];
          mma16<T>(d[m], two_of<T, 0>(lo), two_of<T, 0>(hi), two_of<T, 1>(lo), two_of<T, 1>(hi), x0, x1);
          mma16<T>(d[m], two_of<T, 2>(lo), two_of<T, 2>(hi), two_of<T, 3>(lo), two_of<T, 3>(hi), x2, x3);
        }
        if ((i + 1) % (4 / kGroups) == 0) {  // a group's sums are complete: scaled and added up
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            const int j = i * kGroups / 4 * kRows + r, lane_of = (lane & 28) | (j & 3);
            const float by = scale_of(__shfl_sync(0xffffffffu, s[j / 4], lane_of), p.scale_dtype);
            const float zp = p.zero ? 16.0f + float(__shfl_sync(0xffffffffu, z[j / 4], lane_of) & 15u) : 24.0f;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float& f = d[r >> 1][(r & 1) * 2 + c];
              acc[r >> 1][(r & 1) * 2 + c] += by * (f - zp * sum[c]);
              f = 0.0f;
            }
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) sum[c] = 0.0f;
        }
      }
    }
    __syncwarp();  // the stage may be filled again
    if (++step < p.per) return;
    step = 0;
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
    for (int i = threadIdx.x; i < 16 * kMt * p.M; i += kWarps * 32) {
      // (neighbouring threads: neighbouring rows)
      const int r = i % (16 * kMt), t = i / (16 * kMt), rr = r & 15;
      if (n0 + r < p.N) {
        const float(*part)[128] = sums + (r >> 4) * kWarps;
        const int at = ((rr >> 3) * 2 + (t & 1)) * 32 + (rr & 7) * 4 + (t >> 1);
        float f = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) f += part[w][at];
        static_cast<T*>(const_cast<void*>(p.out.p))[t * p.out.rs + (n0 + r) * p.out.cs] = from_f32<T>(f);
      }
    }
    tile += gridDim.x;
  };
  const int total = mine * p.per;
  for (int it = 0; it < total; it += kStages) {
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
      if (it + i < total) {
        use(i, scale[i], zero[i]);
        load(i, scale[i], zero[i]);
      }
    }
  }
}

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

// 9 to 64 tokens: their words, not the weights, would fill the shared memory's bandwidth if each warp fetched its own.  So
// the warps of a block share the tokens of a unit and take 16 rows each; a cluster of `parts` blocks shares k, and
// adds up its sums through distributed shared memory in a fixed order.
template <typename T, int kGroups, int kNt>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_int4_tokens_kernel(const Int4Params p, const int parts) {
  constexpr int kScales = (2 * kGroups + 3) / 4, kRowsBytes = 16 * 64, kWeightBytes = kWarps * kRowsBytes;
  constexpr int kUnitBytes = kWeightBytes + 8 * kNt * 256;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int rank = int(blockIdx.x) % parts;
  const int64_t n0 = int64_t(blockIdx.x) / parts * (16 * kWarps), row0 = n0 + warp * 16, last = p.N - 1;
  const int u0 = int(int64_t(p.units) * rank / parts), u1 = int(int64_t(p.units) * (rank + 1) / parts);
  const char *rows[2], *scales[kScales];
  const uint8_t* zeros[kScales];
  const int scale_bytes = p.scale_dtype == CCONV_TYPE_FP32 ? 4 : 2;
  auto row_of = [&](int r) { return p.w + min(row0 + r, last) * p.w_rs; };
#pragma unroll
  for (int i = 0; i < 2; ++i) rows[i] = row_of(i * 8 + (lane >> 2));
  // scale number j of a unit: group j / 2, row j % 2; lane q has those with j % 4 = q
#pragma unroll
  for (int i = 0; i < kScales; ++i) {
    const int64_t r = min(row0 + g + 8 * (q % 2), last);
    scales[i] = p.scale + r * p.s_rs * scale_bytes;
    zeros[i] = p.zero + r * p.z_rs;
  }
  uint32_t scale[kStages][kScales], zero[kStages][kScales];
  auto load = [&](int stage, int unit, uint32_t (&s)[kScales], uint32_t (&z)[kScales]) {
    if (unit < u1) {
      const uint32_t to = smem_u32(smem) + stage * kUnitBytes;
      copy_rows(to + warp * kRowsBytes, lane, p, rows, unit, row_of);
      const int64_t k0 = int64_t(unit) * 128 + (lane & 15) * 8;
      const bool there = k0 < p.x_k;
#pragma unroll
      for (int i = 0; i < kNt / 2 + (kNt == 1); ++i) {
        const int t = i * 16 + int(threadIdx.x >> 4);
        if (t < p.M) copy_piece<16>(to + kWeightBytes + token_place(t, (lane & 15) * 16), p.x + t * p.x_rs + (there ? k0 * 2 : 0), there);
      }
#pragma unroll
      for (int i = 0; i < kScales; ++i) {
        const int64_t grp = min(unit * kGroups + (4 * i + q) / 2, p.groups - 1);
        s[i] = load_scale(scales[i], p.scale_dtype, grp * p.s_cs);
        if (p.zero) z[i] = __ldg(zeros[i] + grp * p.z_cs);
      }
    }
    commit_copies();
  };

  start_in_order();
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) load(i, u0 + i, scale[i], zero[i]);
  float acc[kNt][4] = {};
  auto use = [&](int stage, const uint32_t (&s)[kScales], const uint32_t (&z)[kScales]) {
    const uint8_t* const from = smem + stage * kUnitBytes;
    float d[kNt][4] = {};
    uint32_t bias[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i % (4 / kGroups) == 0) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int j = i * kGroups / 4 * 2 + r;
          const uint32_t zp = p.zero ? __shfl_sync(0xffffffffu, z[j / 4], (lane & 28) | (j & 3)) & 15u : 8u;
          bias[r] = High<T>::kBase | zp * 0x10001u;
        }
      }
      uint32_t lo[4], hi[4];
      pairs_of<T>(*reinterpret_cast<const uint32_t*>(from + warp * kRowsBytes + row_place(g, i * 16 + q * 4)), bias[0], lo);
      pairs_of<T>(*reinterpret_cast<const uint32_t*>(from + warp * kRowsBytes + row_place(g + 8, i * 16 + q * 4)), bias[1], hi);
#pragma unroll
      for (int e = 0; e < kNt; ++e) {
        if (8 * e >= p.M) break;
        // (columns behind the last token: whatever lies there, for sums that go nowhere)
        const uint4 v = *reinterpret_cast<const uint4*>(from + kWeightBytes + token_place(8 * e + g, i * 64 + q * 16));
        mma16<T>(d[e], lo[0], hi[0], lo[1], hi[1], v.x, v.y);
        mma16<T>(d[e], lo[2], hi[2], lo[3], hi[3], v.z, v.w);
      }
      if ((i + 1) % (4 / kGroups) == 0) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int j = i * kGroups / 4 * 2 + r;
          const float by = scale_of(__shfl_sync(0xffffffffu, s[j / 4], (lane & 28) | (j & 3)), p.scale_dtype);
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
  };
  for (int u = u0; u < u1; u += kStages) {
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
      if (u + i >= u1) break;
      wait_for_copies<kStages - 2>();
      __syncthreads();  // the unit is there for all, and the one before has been read by all
      constexpr int kBehind = kStages - 1;
      load((i + kBehind) % kStages, u + i + kBehind, scale[(i + kBehind) % kStages], zero[(i + kBehind) % kStages]);
      use(i, scale[i], zero[i]);
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

// The weights as numbers of the operands' type, for products of many tokens: 8 neighbours of a row a thread.
struct ExpandParams {
  const char *w, *scale;
  const uint8_t* zero;
  void* to;
  int64_t w_rs, s_rs, s_cs, z_rs, z_cs, to_rs, N, K;
  int scale_dtype, group;
};
constexpr int kExpandRows = 8;
template <typename T>
__global__ void __launch_bounds__(256) cconv_int4_expand_kernel(const ExpandParams p) {
  start_in_order();
  const int64_t words = (p.K + 7) / 8, i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= words) return;
  const int64_t grp = i * 8 / p.group, last = p.N - 1;
  for (int64_t n0 = int64_t(blockIdx.y) * kExpandRows; n0 < p.N; n0 += int64_t(gridDim.y) * kExpandRows) {
    uint32_t v[kExpandRows], s[kExpandRows], z[kExpandRows];
#pragma unroll
    for (int r = 0; r < kExpandRows; ++r) {
      const int64_t n = min(n0 + r, last);
      v[r] = __ldg(reinterpret_cast<const uint32_t*>(p.w + n * p.w_rs) + i);
      s[r] = load_scale(p.scale, p.scale_dtype, n * p.s_rs + grp * p.s_cs);
      z[r] = p.zero ? __ldg(p.zero + n * p.z_rs + grp * p.z_cs) & 15u : 8u;
    }
#pragma unroll
    for (int r = 0; r < kExpandRows; ++r) {
      if (n0 + r > last) break;
      const float by = scale_of(s[r], p.scale_dtype);
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = by * float(int(v[r] >> (4 * j) & 15u) - int(z[r]));
      T* to = static_cast<T*>(p.to) + (n0 + r) * p.to_rs + i * 8;
      *reinterpret_cast<uint4*>(to) = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
    }
  }
}

template <typename T, int kGroups, int kMt>
cudaError_t launch_rows(const Int4Params& p, int sms, cudaStream_t s) {
  auto f = cconv_int4_kernel<T, kGroups, kMt>;
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, kMt * kWarps * 512 + kWarps * kStages * (16 * kMt * 64 + 8 * 256));
  if (e != cudaSuccess) return e;
  const dim3 grid(unsigned(std::min<int64_t>(cdiv64(p.N, 16 * kMt), 2 * sms)));
  return launch(f, grid, kWarps * 32, size_t(kMt * kWarps * 512 + kWarps * kStages * (16 * kMt * 64 + p.M * 256)), 1, s, p);
}
template <typename T, int kGroups, int kNt>
cudaError_t launch_shared(const Int4Params& p, int sms, cudaStream_t s) {
  auto f = cconv_int4_tokens_kernel<T, kGroups, kNt>;
  constexpr int kSmem = std::max(kStages * (kWarps * 16 * 64 + 8 * kNt * 256), 8 * kNt * (16 * kWarps + 4) * 4);
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, kSmem);
  if (e != cudaSuccess) return e;
  const int64_t tiles = cdiv64(p.N, 16 * kWarps);
  int parts = 1;
  while (parts < 8 && 2 * parts <= p.units && tiles * parts < sms + sms / 2) parts *= 2;
  return launch(f, dim3(unsigned(tiles * parts)), kWarps * 32, kSmem, parts, s, p, parts);
}
template <typename T, int kGroups>
cudaError_t launch_tokens(const Int4Params& p, int sms, cudaStream_t s) {
  if (p.M > 32) return launch_shared<T, kGroups, 8>(p, sms, s);
  if (p.M > 16) return launch_shared<T, kGroups, 4>(p, sms, s);
  if (p.M > 8) return launch_shared<T, kGroups, 2>(p, sms, s);
  // 32 rows a tile where that leaves no SM idle
  return cdiv64(p.N, 32) >= sms ? launch_rows<T, kGroups, 2>(p, sms, s) : launch_rows<T, kGroups, 1>(p, sms, s);
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
  const uintptr_t lies = at | uintptr_t(w_bytes);
  if (M <= kFewTokensInt4) {
    Int4Params p{};
    Mat x(a.x);
    p.x_k = K;
    if (!few_readable(x, M, K, 2)) {
      // (zeros behind a row's end, for k beyond K of its last word)
      const Mat to = st.scratch(M, K, 2);
      p.x_k = to.rs;
      if (K % 8) {
        const int64_t bytes = M * to.rs * 2;
        st.add([=](cudaStream_t s) {
          const cudaError_t e = cudaMemsetAsync(const_cast<void*>(to.p), 0, size_t(bytes), s);
          block_launches() += e == cudaSuccess;
          return block_cuda_error(e, "cconv_int4_product");
        });
      }
      st.copy(x, to, M, K, 2);
      x = to;
    }
    p.x = static_cast<const char*>(x.p);
    p.x_rs = x.rs * 2;
    p.w = static_cast<const char*>(w.p);
    p.w_rs = w.rs;
    p.w_bytes = w_bytes;
    p.scale = static_cast<const char*>(a.scale.data);
    p.s_rs = a.scale.row_stride; p.s_cs = a.scale.col_stride;
    p.zero = static_cast<const uint8_t*>(a.zero.data);
    p.z_rs = a.zero.row_stride; p.z_cs = a.zero.col_stride;
    p.N = N;
    p.M = int(M);
    p.scale_dtype = a.scale_dtype;
    p.piece = (lies & 15) == 0 ? 16 : (lies & 7) == 0 ? 8 : 4;
    p.groups = int(cdiv64(K, group));
    p.units = int(cdiv64(K, 128));
    p.per = int(cdiv64(p.units, kWarps));
    p.out = Mat(a.c);
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
  p.group = group;
  st.add([=](cudaStream_t s) {
    const dim3 grid(unsigned(cdiv64(cdiv64(K, 8), 256)), unsigned(std::min<int64_t>(cdiv64(N, kExpandRows), 65535)));
    return block_cuda_error(dtype == CCONV_TYPE_BF16 ? launch(cconv_int4_expand_kernel<__nv_bfloat16>, grid, 256, 0, 1, s, p)
                                                     : launch(cconv_int4_expand_kernel<__half>, grid, 256, 0, 1, s, p),
                            "cconv_int4_expand_kernel");
  });
  Launch l;
  l.epilogue = kStore;
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
