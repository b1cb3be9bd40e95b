// A mixture-of-experts layer for a few tokens: each token goes through the k experts that its router scores
// highest, and their results are added up with softmax weights.
//
//   logits = x Wr^T,  e_j: the k largest (of equal ones the first),  p = softmax of them or, not normalised, of all
//   h = act(x Wg_e^T) * (x Wu_e^T),  y = sum_j p_j h Wd_{e_j}^T
//
// What bounds it is HBM: the weights of the experts in use, each read once for all tokens that chose it.  Three
// launches, which follow one another without a gap (a kernel is put in place while the one in front ends):
//   router   one cluster of eight blocks for 64 tokens: logits, a barrier, the choice
//   gate/up  tiles of 8 hidden channels of an expert in use, its tokens gathered as columns; h in two 16-bit parts,
//            whose sum has twice the type's precision
//   down     tiles of 16 or 8 channels through all experts in use; a column is a token, so that the weighted sums of
//            all its experts stay in one accumulator, added up in the order of the experts
// Both weight kernels build the lists of who goes where themselves from the choice (a microsecond less than to wait
// for a kernel that would), stream weights through rings in shared memory, one a warp, and multiply by warp-wide
// matrix instructions (m16n8): tcgen05 would want tiles that a few tokens leave almost empty.
#include "block_moe.h"

#include <algorithm>
#include <type_traits>

#include "block_device.cuh"
#include "block_few.h"
#include "block_launch.h"
#include "block_mma.cuh"
#include "block_steps.h"
#include "ptx_sm100.cuh"

namespace cconv {
namespace {

constexpr int kTokens = 64;  // of a launch of the weight kernels
constexpr int kWarps = 8, kStages = 4, kUnitBytes = 2048;
constexpr int kRouterBlocks = 8, kRouterWarps = 16;

struct MoeParams {
  const char* x;     // tokens, rows of x_k elements that may be read
  int64_t x_rs, x_k;  // bytes; elements, a multiple of 8
  int64_t D, F;
  int T, E, k, act, dtype, normalize;
  const char* router;  // rows readable like x's
  int64_t router_rs;
  float* logits;       // [T][E]
  int* ids; int64_t ids_rs, ids_cs;
  float* weights; int64_t weights_rs, weights_cs;
  // expert matrices: element strides
  const char *w_gate, *w_up, *w_down;
  int64_t gate_es, gate_rs, gate_cs, up_es, up_rs, up_cs, down_es, down_rs, down_cs;
  int piece_in, piece_out;  // bytes that rows of gate and up, and of down, can be copied in (2: element by element)
  char *h, *h_lo;           // [T k][h_rs] elements
  int64_t h_rs;
  Mat out;
};

// ---- router --------------------------------------------------------------------------------------
// Order of scores: larger first, then the lower index; NaN last.
__device__ __forceinline__ uint64_t rank_of(float v, int e) {
  const uint32_t b = __float_as_uint(v);
  const uint32_t up = v != v ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return uint64_t(up) << 32 | uint32_t(~e);
}
__device__ __forceinline__ uint64_t warp_max(uint64_t v) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, uint32_t(v >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, uint32_t(v >> 32) == hi ? uint32_t(v) : 0u);
  return uint64_t(hi) << 32 | lo;
}

// Experts are dealt to the blocks of the cluster in neighbouring ranges; a block's warps share the channels.  Then each
// warp of the cluster chooses for tokens of its own.
template <typename T, int kNt>
__global__ void __launch_bounds__(kRouterWarps * 32) cconv_moe_router_kernel(const MoeParams p) {
  __shared__ float sums[kRouterWarps][128];
  start_in_order();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int rank = int(cluster_ctarank()), t0 = int(blockIdx.x / kRouterBlocks) * kTokens, tokens = min(kTokens, p.T - t0);
  const int per = (p.E + kRouterBlocks - 1) / kRouterBlocks, e0 = rank * per, e1 = min(p.E, e0 + per);
  for (int m = e0; m < e1; m += 16) {
    const char* r0 = p.router + int64_t(min(m + g, p.E - 1)) * p.router_rs;
    const char* r1 = p.router + int64_t(min(m + g + 8, p.E - 1)) * p.router_rs;
    float acc[kNt][4] = {};
    const int64_t units = (p.x_k + 31) / 32;
#pragma unroll 2
    for (int64_t u = warp; u < units; u += kRouterWarps) {
      const int64_t k0 = u * 32 + q * 8;
      const bool in = k0 < p.x_k;
      const uint4 none = make_uint4(0, 0, 0, 0);
      const uint4 a0 = in ? *reinterpret_cast<const uint4*>(r0 + k0 * 2) : none;
      const uint4 a1 = in ? *reinterpret_cast<const uint4*>(r1 + k0 * 2) : none;
#pragma unroll
      for (int e = 0; e < kNt; ++e) {
        const int t = 8 * e + g;
        const uint4 v = in && t < tokens ? *reinterpret_cast<const uint4*>(p.x + int64_t(t0 + t) * p.x_rs + k0 * 2) : none;
        mma16<T>(acc[e], a0.x, a1.x, a0.y, a1.y, v.x, v.y);
        mma16<T>(acc[e], a0.z, a1.z, a0.w, a1.w, v.z, v.w);
      }
    }
#pragma unroll
    for (int e = 0; e < kNt; ++e) {
      if (8 * e >= tokens) break;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[warp][i * 32 + lane] = acc[e][i];
      __syncthreads();
      if (threadIdx.x < 128) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kRouterWarps; ++w) s += sums[w][threadIdx.x];
        const int i = threadIdx.x >> 5;
        const int row = m + g + (i >> 1) * 8, t = 8 * e + 2 * q + (i & 1);
        if (row < e1 && t < tokens) p.logits[int64_t(t0 + t) * p.E + row] = s;
      }
    }
  }
  cluster_sync_all();
  for (int t = rank * kRouterWarps + warp; t < tokens; t += kRouterBlocks * kRouterWarps) {
    const float* row = p.logits + int64_t(t0 + t) * p.E;
    uint64_t before = ~uint64_t(0);
    float mine = 0.0f, largest = 0.0f;  // lane j: the j-th choice's score
    int id = 0;
    for (int j = 0; j < p.k; ++j) {
      uint64_t best = 0;
      for (int e = lane; e < p.E; e += 32) {
        const uint64_t r = rank_of(row[e], e);
        if (r < before && r > best) best = r;
      }
      before = warp_max(best);
      const int e = int(~uint32_t(before));
      const float score = row[e];
      if (j == 0) largest = score;
      if (lane == j) mine = score, id = e;
    }
    float sum = 0.0f;
    if (p.normalize) {
      sum = lane < p.k ? expf(mine - largest) : 0.0f;
    } else {
      for (int e = lane; e < p.E; e += 32) sum += expf(row[e] - largest);
    }
    sum = warp_sum(sum);
    if (lane < p.k) {
      p.ids[int64_t(t0 + t) * p.ids_rs + lane * p.ids_cs] = id;
      p.weights[int64_t(t0 + t) * p.weights_rs + lane * p.weights_cs] = __fdiv_rn(expf(mine - largest), sum);
    }
  }
}

// ---- who goes where --------------------------------------------------------------------------------
// Of the tokens of a launch, in shared memory: the experts in use in ascending order, each with the set of its tokens
// and where their pairs (token, choice) begin in `pairs`, ascending by token.  An expert that a token names twice counts
// once, with both weights; numbers that are no expert's count for nothing.
struct Routes {
  uint64_t* tokens;   // [used]: bit t
  uint16_t* expert;   // [used]
  uint16_t* first;    // [used]
  uint16_t* pairs;    // [pairs]: t k + j
  float* weight;      // [t k + j] (down kernel)
  int used;
};
constexpr int routes_bytes(int E, int pairs, bool weights) {
  return E * 8 + E * 4 + (pairs + 1) / 2 * 4 + (weights ? pairs * 4 : 0);
}

template <bool kWeights>
__device__ __forceinline__ Routes routes_of(const MoeParams& p, uint8_t* smem, int* scratch) {
  const int E = p.E, pairs = p.T * p.k, tid = threadIdx.x, nt = kWarps * 32;
  Routes r;
  r.tokens = reinterpret_cast<uint64_t*>(smem);
  r.weight = reinterpret_cast<float*>(r.tokens + E);
  r.expert = reinterpret_cast<uint16_t*>(r.weight + (kWeights ? pairs : 0));
  r.first = r.expert + E;
  r.pairs = r.first + E;
  for (int e = tid; e < E; e += nt) r.tokens[e] = 0;
  __syncthreads();
  auto id_of = [&](int t, int j) { return __ldg(p.ids + t * p.ids_rs + j * p.ids_cs); };
  for (int i = tid; i < pairs; i += nt) {
    const int t = i / p.k, e = id_of(t, i - t * p.k);
    if (e >= 0 && e < E) atomicOr(reinterpret_cast<unsigned long long*>(r.tokens + e), 1ull << t);
  }
  __syncthreads();
  // places of the experts in use: at most 1024 experts, 4 a thread, all threads' counts added up by the warps
  uint64_t mine[4];
  int n = 0, entries = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = tid * 4 + i;
    mine[i] = e < E ? r.tokens[e] : 0;
    n += mine[i] != 0;
    entries += __popcll(mine[i]);
  }
  int both = n | entries << 16, incl = both;  // (at most 1024 and 2048)
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if ((tid & 31) >= o) incl += v;
  }
  if ((tid & 31) == 31) scratch[tid >> 5] = incl;
  __syncthreads();
  int base = incl - both, total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < (tid >> 5)) base += scratch[w];
    total += scratch[w];
  }
  r.used = total & 0xffff;
  int at = base & 0xffff, first = base >> 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (mine[i] == 0) continue;
    r.tokens[at] = mine[i];  // (every thread has read its own; at <= its first)
    r.expert[at] = uint16_t(tid * 4 + i);
    r.first[at] = uint16_t(first);
    ++at;
    first += __popcll(mine[i]);
  }
  __syncthreads();
  for (int i = tid; i < pairs; i += nt) {
    const int t = i / p.k, j = i - t * p.k, e = id_of(t, j);
    if (e < 0 || e >= E) continue;
    bool again = false;
    for (int o = 0; o < j; ++o) again |= id_of(t, o) == e;
    if (again) continue;
    int lo = 0, hi = r.used - 1;  // e's place
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (r.expert[mid] < e) lo = mid + 1;
      else hi = mid;
    }
    r.pairs[r.first[lo] + __popcll(r.tokens[lo] & ((1ull << t) - 1))] = uint16_t(i);
    if (kWeights) {
      float w = 0.0f;
      for (int o = j; o < p.k; ++o)
        if (id_of(t, o) == e) w += __ldg(p.weights + t * p.weights_rs + o * p.weights_cs);
      r.weight[i] = w;
    }
  }
  __syncthreads();
  return r;
}

// ---- weights through a ring -------------------------------------------------------------------------
// A unit is 16 segments of 128 bytes; segments of odd number have their halves swapped, so that the 16-byte words that
// eight lanes read together lie in different banks.
__device__ __forceinline__ uint32_t place(int segment, int byte) { return segment * 128 + (byte ^ ((segment & 1) << 6)); }

// Copies a unit: segment s is 64 elements from at(s), of which those before left(s) are there and the others zeros.
template <int kBytes, typename At, typename Left>
__device__ __forceinline__ void copy_unit_by(uint32_t to, int lane, At at, Left left) {
  constexpr int kAcross = 128 / kBytes;
#pragma unroll
  for (int i = 0; i < kUnitBytes / 32 / kBytes; ++i) {
    const int c = i * 32 + lane, seg = c / kAcross, off = c % kAcross * kBytes;
    const char* from = at(seg);
    const bool there = off < left(seg) * 2;
    const uint32_t n = there ? kBytes : 0;
    if constexpr (kBytes == 16)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + place(seg, off)), "l"(there ? from + off : from), "r"(n) : "memory");
    else
      asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to + place(seg, off)), "l"(there ? from + off : from), "n"(kBytes), "r"(n) : "memory");
  }
}
template <typename At, typename Left, typename Step>
__device__ __forceinline__ void copy_unit(uint8_t* ring, int piece, int lane, At at, Left left, Step step) {
  const uint32_t to = smem_u32(ring);
  if (piece == 16) {
    copy_unit_by<16>(to, lane, at, left);
  } else if (piece == 4) {
    copy_unit_by<4>(to, lane, at, left);
  } else {
    // element by element, step(s) apart
    for (int seg = 0; seg < 16; ++seg) {
      const uint16_t* from = reinterpret_cast<const uint16_t*>(at(seg));
      const int64_t n = left(seg), cs = step(seg);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int e = i * 32 + lane;
        *reinterpret_cast<uint16_t*>(ring + place(seg, e * 2)) = e < n ? __ldg(from + e * cs) : uint16_t(0);
      }
    }
  }
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void wait_for_unit() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
  __syncwarp();
}
__device__ __forceinline__ uint4 load_16(const char* p) { return *reinterpret_cast<const uint4*>(p); }

// ---- gate and up ------------------------------------------------------------------------------------
// Block b takes the items b, b + gridDim.x, ... of (expert in use, 8 hidden channels); its warps share the channels in
// units of 64.  Rows 0 to 7 of a tile are the gate's, rows 8 to 15 the up projection's.
template <typename T, int kNt>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_moe_gate_up_kernel(const MoeParams p) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int scratch[kWarps];
  float(*const sums)[128] = reinterpret_cast<float(*)[128]>(smem + kWarps * kStages * kUnitBytes);  // [kNt * kWarps]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  uint8_t* const ring = smem + warp * (kStages * kUnitBytes);
  start_in_order();
  const Routes r = routes_of<false>(p, smem + kWarps * (kStages * kUnitBytes + kNt * 512), scratch);
  const int tiles = int((p.F + 7) / 8);
  const int units = int((p.D + 63) / 64), per = (units + kWarps - 1) / kWarps, u0 = warp * per;
  const int64_t items = int64_t(r.used) * tiles, stride = gridDim.x;
  const int64_t mine = int64_t(blockIdx.x) < items ? (items - 1 - blockIdx.x) / stride + 1 : 0;

  // (an item's place and tile, kept without divisions)
  const int step_place = int(stride / tiles), step_tile = int(stride % tiles);
  int lplace = int(blockIdx.x / tiles), ltile = int(blockIdx.x % tiles), lu = 0;
  auto load = [&](int stage) {
    const int unit = u0 + lu;
    if (lplace < r.used && unit < units) {
      const int64_t e = r.expert[lplace], k0 = int64_t(unit) * 64;
      copy_unit(ring + stage * kUnitBytes, p.piece_in, lane, [&](int seg) {
        const int64_t f = min(int64_t(ltile) * 8 + (seg & 7), p.F - 1);
        return seg < 8 ? p.w_gate + (e * p.gate_es + f * p.gate_rs + k0 * p.gate_cs) * 2
                       : p.w_up + (e * p.up_es + f * p.up_rs + k0 * p.up_cs) * 2;
      }, [&](int) { return p.D - k0; }, [&](int seg) { return seg < 8 ? p.gate_cs : p.up_cs; });
    }
    commit_copies();
    if (++lu == per) {
      lu = 0;
      ltile += step_tile;
      lplace += step_place;
      if (ltile >= tiles) ltile -= tiles, ++lplace;
    }
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) load(i);

  int pl = int(blockIdx.x / tiles), tile = int(blockIdx.x % tiles), step = 0;
  float acc[kNt][4] = {};
  const char* row[kNt];  // the tokens of this lane's columns
  int count = 0, first = 0;
  auto start_item = [&]() {
    count = __popcll(r.tokens[pl]);
    first = r.first[pl];
#pragma unroll
    for (int e = 0; e < kNt; ++e) row[e] = p.x + int64_t(r.pairs[first + min(8 * e + g, count - 1)] / p.k) * p.x_rs + q * 16;
  };
  auto use = [&](int stage) {
    if (step == 0) start_item();
    const int unit = u0 + step;
    wait_for_unit();
    if (unit < units) {
      const uint8_t* from = ring + stage * kUnitBytes;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t k0 = int64_t(unit) * 64 + i * 32;
        const uint4 a0 = *reinterpret_cast<const uint4*>(from + place(g, i * 64 + q * 16));
        const uint4 a1 = *reinterpret_cast<const uint4*>(from + place(g + 8, i * 64 + q * 16));
#pragma unroll
        for (int e = 0; e < kNt; ++e) {
          if (8 * e >= count) break;
          uint4 v = make_uint4(0, 0, 0, 0);
          if (8 * e + g < count && k0 + q * 8 < p.x_k) v = load_16(row[e] + k0 * 2);
          mma16<T>(acc[e], a0.x, a1.x, a0.y, a1.y, v.x, v.y);
          mma16<T>(acc[e], a0.z, a1.z, a0.w, a1.w, v.z, v.w);
        }
      }
    }
    __syncwarp();
    if (++step < per) return;
    step = 0;
    __syncthreads();  // the sums before have been read
#pragma unroll
    for (int e = 0; e < kNt; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (8 * e < count) sums[e * kWarps + warp][i * 32 + lane] = acc[e][i];
        acc[e][i] = 0.0f;
      }
    __syncthreads();
    for (int i = threadIdx.x; i < 8 * count; i += kWarps * 32) {
      const int f = i & 7, c = i >> 3, at = (c & 1) * 32 + f * 4 + ((c & 7) >> 1);
      const float(*part)[128] = sums + (c >> 3) * kWarps;
      float a[1] = {0.0f}, u[1] = {0.0f};
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        a[0] += part[w][at];
        u[0] += part[w][at + 64];
      }
      gate(p.act, a, u);
      const int64_t channel = int64_t(tile) * 8 + f, to = int64_t(r.pairs[first + c]) * p.h_rs + channel;
      if (channel >= p.F) a[0] = 0.0f;  // the rest of the row's last 16 bytes
      const T hi = from_f32<T>(a[0]);
      reinterpret_cast<T*>(p.h)[to] = hi;
      // (what overflows has no second part)
      reinterpret_cast<T*>(p.h_lo)[to] = from_f32<T>(isfinite(to_f32(hi)) ? a[0] - to_f32(hi) : 0.0f);
    }
    tile += step_tile;
    pl += step_place;
    if (tile >= tiles) tile -= tiles, ++pl;
  };
  const int64_t total = mine * per;
  int stage = 0;
  for (int64_t it = 0; it < total; ++it) {
    use(stage);
    load(stage);
    stage = (stage + 1) % kStages;
  }
}

// ---- down -------------------------------------------------------------------------------------------
// Block b takes the tiles b, b + gridDim.x, ... of kRows channels, each through all experts in use; its warps share
// the hidden channels in units of 64 (16 rows) or 128 (8 rows, whose second halves are segments 8 to 15).
template <typename T, int kNt, int kRows>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_moe_down_kernel(const MoeParams p, const int early) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int scratch[kWarps];
  float(*const sums)[128] = reinterpret_cast<float(*)[128]>(smem + kWarps * kStages * kUnitBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  uint8_t* const ring = smem + warp * (kStages * kUnitBytes);
  constexpr int kUnit = kRows == 16 ? 64 : 128;
  const int tiles = int((p.D + kRows - 1) / kRows);
  const int units = int((p.F + kUnit - 1) / kUnit), per = (units + kWarps - 1) / kWarps, u0 = warp * per;

  // Behind the gate and up kernel of the same call, which lets this one in only once everything before the call and the
  // router are complete, the choice and the weights are there already; h is waited for below.
  if (!early) start_in_order();
  const Routes r = routes_of<true>(p, smem + kWarps * (kStages * kUnitBytes + kNt * 512), scratch);
  int lt = blockIdx.x, lplace = 0, lu = 0;
  auto load = [&](int stage) {
    const int unit = u0 + lu;
    if (lt < tiles && lplace < r.used && unit < units) {
      const int64_t e = r.expert[lplace], k0 = int64_t(unit) * kUnit;
      auto part = [&](int seg) { return k0 + (kRows == 8 ? seg >> 3 << 6 : 0); };
      copy_unit(ring + stage * kUnitBytes, p.piece_out, lane, [&](int seg) {
        const int64_t d = min(int64_t(lt) * kRows + (seg & (kRows - 1)), p.D - 1), k = part(seg);
        return p.w_down + (e * p.down_es + d * p.down_rs + (k < p.F ? k : 0) * p.down_cs) * 2;
      }, [&](int seg) { return p.F - part(seg); }, [&](int) { return p.down_cs; });
    }
    commit_copies();
    if (++lu == per) {
      lu = 0;
      if (++lplace >= r.used) lplace = 0, lt += gridDim.x;
    }
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) load(i);
  if (early) start_in_order();

  int pl = 0, step = 0;
  float acc[kNt][4] = {}, d[kNt][4] = {};
  int64_t row[kNt];  // where h of this lane's tokens begins; -1: they have not chosen the expert
  uint64_t tokens = 0;
  int first = 0;
  auto pair_of_token = [&](int t) { return r.pairs[first + __popcll(tokens & ((1ull << t) - 1))]; };
  auto use = [&](int stage) {
    if (step == 0) {
      tokens = r.tokens[pl];
      first = r.first[pl];
#pragma unroll
      for (int e = 0; e < kNt; ++e) {
        const int t = 8 * e + g;
        row[e] = tokens >> t & 1 ? int64_t(pair_of_token(t)) * p.h_rs * 2 + q * 16 : -1;
      }
    }
    const int unit = u0 + step;
    wait_for_unit();
    if (unit < units) {
      const uint8_t* from = ring + stage * kUnitBytes;
#pragma unroll
      for (int i = 0; i < kUnit / 32; ++i) {
        const int64_t k0 = int64_t(unit) * kUnit + i * 32;
        uint4 a0, a1;
        if constexpr (kRows == 16) {
          a0 = *reinterpret_cast<const uint4*>(from + place(g, i * 64 + q * 16));
          a1 = *reinterpret_cast<const uint4*>(from + place(g + 8, i * 64 + q * 16));
        } else {
          a0 = *reinterpret_cast<const uint4*>(from + place(g + (i >> 1) * 8, (i & 1) * 64 + q * 16));
          a1 = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < kNt; ++e) {
          if ((tokens >> (8 * e) & 0xff) == 0) continue;
          uint4 v = make_uint4(0, 0, 0, 0), w = v;
          if (row[e] >= 0 && k0 + q * 8 < p.h_rs) {
            v = load_16(p.h + row[e] + k0 * 2);
            w = load_16(p.h_lo + row[e] + k0 * 2);
          }
          mma16<T>(d[e], a0.x, a1.x, a0.y, a1.y, v.x, v.y);
          mma16<T>(d[e], a0.z, a1.z, a0.w, a1.w, v.z, v.w);
          mma16<T>(d[e], a0.x, a1.x, a0.y, a1.y, w.x, w.y);
          mma16<T>(d[e], a0.z, a1.z, a0.w, a1.w, w.z, w.w);
        }
      }
    }
    __syncwarp();
    if (++step < per) return;
    step = 0;
    // the expert's share, times the weights of this lane's columns
#pragma unroll
    for (int e = 0; e < kNt; ++e) {
      if ((tokens >> (8 * e) & 0xff) == 0) continue;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int t = 8 * e + 2 * q + c;
        if (tokens >> t & 1) {
          const float w = r.weight[pair_of_token(t)];
          acc[e][c] += w * d[e][c];
          acc[e][2 + c] += w * d[e][2 + c];
        }
        d[e][c] = d[e][2 + c] = 0.0f;
      }
    }
    ++pl;
  };
  int stage = 0;
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    pl = 0;
    const int total = r.used * per;
    for (int it = 0; it < total; ++it) {
      use(stage);
      load(stage);
      stage = (stage + 1) % kStages;
    }
    __syncthreads();  // the sums before have been read
#pragma unroll
    for (int e = 0; e < kNt; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sums[e * kWarps + warp][i * 32 + lane] = acc[e][i];
        acc[e][i] = 0.0f;
      }
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * p.T; i += kWarps * 32) {
      const int rr = i % kRows, t = i / kRows;
      const int64_t channel = int64_t(tile) * kRows + rr;
      if (channel >= p.D) continue;
      const int at = ((rr >> 3) * 2 + (t & 1)) * 32 + (rr & 7) * 4 + ((t & 7) >> 1);
      const float(*part)[128] = sums + (t >> 3) * kWarps;
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) s += part[w][at];
      static_cast<T*>(const_cast<void*>(p.out.p))[t * p.out.rs + channel * p.out.cs] = from_f32<T>(s);
    }
  }
}

// ---- launches ---------------------------------------------------------------------------------------
template <typename T, int kNt>
cudaError_t launch_router(const MoeParams& p, cudaStream_t s) {
  const dim3 grid(unsigned(cdiv64(p.T, kTokens) * kRouterBlocks));
  return launch(cconv_moe_router_kernel<T, kNt>, grid, kRouterWarps * 32, 0, kRouterBlocks, s, p);
}

constexpr int kRing = kWarps * kStages * kUnitBytes;
int smem_of(const MoeParams& p, int nt, bool weights) { return kRing + kWarps * nt * 512 + routes_bytes(p.E, p.T * p.k, weights); }
constexpr int kMostSmem = kRing + kWarps * 8 * 512 + routes_bytes(int(kMostExperts), kTokens * int(kMostChosen), true);

template <typename T, int kNt>
cudaError_t launch_gate_up(const MoeParams& p, int sms, cudaStream_t s) {
  auto f = cconv_moe_gate_up_kernel<T, kNt>;
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, kMostSmem);
  if (e != cudaSuccess) return e;
  const int64_t most = std::min<int64_t>(p.E, int64_t(p.T) * p.k) * cdiv64(p.F, 8);
  return launch(f, dim3(unsigned(std::min<int64_t>(most, 2 * sms))), kWarps * 32, smem_of(p, kNt, false), 1, s, p);
}
template <typename T, int kNt, int kRows>
cudaError_t launch_down_rows(const MoeParams& p, int sms, cudaStream_t s) {
  auto f = cconv_moe_down_kernel<T, kNt, kRows>;
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, kMostSmem);
  if (e != cudaSuccess) return e;
  return launch(f, dim3(unsigned(std::min<int64_t>(cdiv64(p.D, kRows), 2 * sms))), kWarps * 32, smem_of(p, kNt, true), 1, s, p, 1);
}
template <typename T, int kNt>
cudaError_t launch_down(const MoeParams& p, int sms, cudaStream_t s) {
  // 16 rows a tile where that leaves no SM with less than two blocks
  return cdiv64(p.D, 16) >= 2 * sms ? launch_down_rows<T, kNt, 16>(p, sms, s) : launch_down_rows<T, kNt, 8>(p, sms, s);
}
// Calls f(T(), columns of 8) for the call's type and T tokens, at most 64.
template <typename F>
cudaError_t with_columns(int dtype, int64_t T, F f) {
  auto columns = [&](auto type) {
    if (T <= 8) return f(type, std::integral_constant<int, 1>());
    if (T <= 16) return f(type, std::integral_constant<int, 2>());
    if (T <= 32) return f(type, std::integral_constant<int, 4>());
    return f(type, std::integral_constant<int, 8>());
  };
  return dtype == CCONV_TYPE_BF16 ? columns(__nv_bfloat16()) : columns(__half());
}

// Bytes that rows of an expert's matrix can be copied in.
int piece_of(const cconv_matrix& m, int64_t expert_stride, int64_t rows, int64_t cols, int64_t experts) {
  if (m.col_stride != 1 && cols > 1) return 2;
  const uintptr_t lies = reinterpret_cast<uintptr_t>(m.data) | uintptr_t(rows > 1 ? m.row_stride * 2 : 0) |
                         uintptr_t(experts > 1 ? expert_stride * 2 : 0) | uintptr_t(cols * 2);
  return (lies & 15) == 0 ? 16 : (lies & 3) == 0 ? 4 : 2;
}

// Rows that 16 bytes at a time can be read from, with zeros behind K; *k: elements that may be read.
Mat padded(Steps& st, const cconv_matrix& m, int64_t rows, int64_t K, int64_t* k) {
  *k = K;
  if (few_readable(Mat(m), rows, K, 2)) return Mat(m);
  const Mat to = st.scratch(rows, K, 2);
  *k = to.rs;
  if (K % 8) {
    const int64_t bytes = rows * to.rs * 2;
    st.add([=](cudaStream_t s) {
      const cudaError_t e = cudaMemsetAsync(const_cast<void*>(to.p), 0, size_t(bytes), s);
      block_launches() += e == cudaSuccess;
      return block_cuda_error(e, "cconv_moe_forward");
    });
  }
  st.copy(Mat(m), to, rows, K, 2);
  return to;
}

void plan(Steps& st, const cconv_moe_args& a) {
  const int sms = st.sms();
  MoeParams p{};
  const Mat x = padded(st, a.x, a.T, a.D, &p.x_k);
  p.x = static_cast<const char*>(x.p);
  p.x_rs = x.rs * 2;
  p.D = a.D;
  p.F = a.F;
  p.E = int(a.E);
  p.k = a.top_k;
  p.act = a.act;
  p.dtype = a.dtype;
  p.normalize = a.normalize;
  p.ids = static_cast<int*>(a.ids.data); p.ids_rs = a.ids.row_stride; p.ids_cs = a.ids.col_stride;
  p.weights = static_cast<float*>(a.weights.data); p.weights_rs = a.weights.row_stride; p.weights_cs = a.weights.col_stride;
  p.w_gate = static_cast<const char*>(a.w_gate.data);
  p.w_up = static_cast<const char*>(a.w_up.data);
  p.w_down = static_cast<const char*>(a.w_down.data);
  p.gate_es = a.gate_stride; p.gate_rs = a.w_gate.row_stride; p.gate_cs = a.w_gate.col_stride;
  p.up_es = a.up_stride; p.up_rs = a.w_up.row_stride; p.up_cs = a.w_up.col_stride;
  p.down_es = a.down_stride; p.down_rs = a.w_down.row_stride; p.down_cs = a.w_down.col_stride;
  p.piece_in = std::min(piece_of(a.w_gate, a.gate_stride, a.F, a.D, a.E), piece_of(a.w_up, a.up_stride, a.F, a.D, a.E));
  p.piece_out = piece_of(a.w_down, a.down_stride, a.D, a.F, a.E);
  const int64_t chunk = std::min<int64_t>(a.T, kTokens);
  const Mat h = st.scratch(chunk * a.top_k, a.F, 2), h_lo = st.scratch(chunk * a.top_k, a.F, 2);
  p.h = static_cast<char*>(const_cast<void*>(h.p));
  p.h_lo = static_cast<char*>(const_cast<void*>(h_lo.p));
  p.h_rs = h.rs;
  p.out = Mat(a.out);
  if (a.router.data) {
    int64_t k = 0;
    const Mat router = padded(st, a.router, a.E, a.D, &k);
    p.router = static_cast<const char*>(router.p);
    p.router_rs = router.rs * 2;
    p.logits = static_cast<float*>(const_cast<void*>(st.scratch(a.T, a.E, 4).p));
    MoeParams r = p;
    r.T = int(a.T);
    st.add([=](cudaStream_t s) {
      return block_cuda_error(with_columns(r.dtype, r.T, [&](auto type, auto nt) { return launch_router<decltype(type), decltype(nt)::value>(r, s); }),
                              "cconv_moe_router_kernel");
    });
  }
  for (int64_t t0 = 0; t0 < a.T && a.F; t0 += kTokens) {
    MoeParams c = p;
    c.T = int(std::min<int64_t>(kTokens, a.T - t0));
    c.x += t0 * c.x_rs;
    c.ids += t0 * c.ids_rs;
    c.weights += t0 * c.weights_rs;
    c.out.p = static_cast<const char*>(c.out.p) + t0 * c.out.rs * 2;
    st.add([=](cudaStream_t s) {
      cudaError_t e = with_columns(c.dtype, c.T, [&](auto type, auto nt) { return launch_gate_up<decltype(type), decltype(nt)::value>(c, sms, s); });
      if (e == cudaSuccess)
        e = with_columns(c.dtype, c.T, [&](auto type, auto nt) { return launch_down<decltype(type), decltype(nt)::value>(c, sms, s); });
      return block_cuda_error(e, "cconv_moe_forward");
    });
  }
}

}  // namespace

int64_t moe_workspace(const cconv_moe_args& a, int sms) {
  Steps st(nullptr, sms, 2, a.dtype);
  plan(st, a);
  return st.bytes();
}

int run_moe(const cconv_moe_args& a, int sms, cudaStream_t s) {
  Steps st(a.workspace, sms, 2, a.dtype);
  plan(st, a);
  return st.run(s);
}

}  // namespace cconv
