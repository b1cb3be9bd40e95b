// A mixture-of-experts layer for a few tokens: each token goes through the k experts that its router scores
// highest, and their results are added up with softmax weights.
//
//   logits = x Wr^T,  e_j: the k largest (of equal ones the first),  p = softmax of them or, not normalised, of all
//   h = act(x Wg_e^T) * (x Wu_e^T),  y = sum_j p_j h Wd_{e_j}^T
//
// What bounds it is HBM: the weights of the experts in use, each read once for all tokens that chose it.  Three
// launches, which follow one another without a gap (a kernel is put in place while the one in front ends):
//   router   one cluster of eight blocks for 64 tokens: scores, a barrier, the choice
//   gate/up  tiles of 8 hidden channels of an expert in use, its tokens gathered as columns, 8 or 16 at a time; h in
//            two 16-bit parts, whose sum has twice the type's precision
//   down     tiles of 16 channels through all experts in use, in one block or shared by a cluster
// Both weight kernels build the lists of who goes where themselves from the choice (a microsecond less than to wait
// for a kernel that would), stream weights through rings in shared memory, one a warp, and multiply by warp-wide
// matrix instructions (m16n8): tcgen05 would want tiles that a few tokens leave almost empty.
#include "block_moe.h"

#include <algorithm>
#include <type_traits>

#include "block_device.cuh"
#include "block_launch.h"
#include "block_mma.cuh"
#include "block_pad.h"
#include "block_steps.h"
#include "ptx_sm100.cuh"

namespace cconv {
namespace {

constexpr int kTokens = 64;  // of a launch of the weight kernels
constexpr int kWarps = 8;
constexpr int kRouterBlocks = 8, kRouterWarps = 16;

struct MoeParams {
  const char* x;     // tokens, rows of x_k elements that may be read
  int64_t x_rs, x_k;  // bytes; elements, a multiple of 8
  int64_t D, F;
  int T, E, k, act, dtype, normalize;
  const char* router;  // rows readable like x's
  int64_t router_rs;
  int* ids; int64_t ids_rs, ids_cs;
  float* weights; int64_t weights_rs, weights_cs;
  // expert matrices: element strides
  const char *w_gate, *w_up, *w_down;
  int64_t gate_es, gate_rs, gate_cs, up_es, up_rs, up_cs, down_es, down_rs, down_cs;
  int piece_in, piece_out;  // of gate and up, and of down: see piece_of
  char *h, *h_lo;           // [T k][h_rs] elements
  int64_t h_rs;
  Mat out;
};

__device__ __forceinline__ uint4 load_16(const char* p) { return *reinterpret_cast<const uint4*>(p); }

// ---- router --------------------------------------------------------------------------------------
// A score as a number of the same order, NaN below all others; 0 is none.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t b = __float_as_uint(v);
  return v != v ? 1u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float score_of(uint32_t key) {  // (key 1: a NaN too)
  return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}

// Channels are dealt to the blocks of the cluster, and a block's share of them and 16 experts at a time to its warps:
// with the usual sizes a warp's loads are all on their way at once.  Partial scores [slice][token][expert] lie in
// shared memory; a block adds its own up and sends them to the block that chooses for the token (t % 8), whose warps
// add up the blocks' [block][t / 8][expert].
template <typename T, int kNt>
__global__ void __launch_bounds__(kRouterWarps * 32) cconv_moe_router_kernel(const MoeParams p, const int chunk) {
  extern __shared__ __align__(128) uint8_t smem[];
  float* const part = reinterpret_cast<float*>(smem);
  cluster_arrive();
  start_in_order();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int rank = int(cluster_ctarank()), t0 = int(blockIdx.x / kRouterBlocks) * chunk, tokens = min(chunk, p.T - t0);
  const int groups = (p.E + 15) / 16, slices = groups >= kRouterWarps ? 1 : kRouterWarps / groups;
  const int units = int((p.x_k + 31) / 32), all = slices * kRouterBlocks, slice = warp / groups;
  if (slice < slices) {
    // of the cluster's slices, this warp's
    const int mine = rank * slices + slice, u0 = int(int64_t(units) * mine / all), u1 = int(int64_t(units) * (mine + 1) / all);
    for (int m = slices == 1 ? warp : warp % groups; m < groups; m += kRouterWarps) {
      const char* r0 = p.router + int64_t(min(16 * m + g, p.E - 1)) * p.router_rs;
      const char* r1 = p.router + int64_t(min(16 * m + g + 8, p.E - 1)) * p.router_rs;
      float acc[kNt][4] = {};
      // kBatch units at once: with the usual sizes they are all that the warp has, and wait for memory together
      constexpr int kBatch = kNt == 1 ? 4 : kNt <= 4 ? 2 : 1;
      const uint4 none = make_uint4(0, 0, 0, 0);
      for (int first = u0; first < u1; first += kBatch) {
        uint4 a0[kBatch], a1[kBatch], v[kBatch][kNt];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int64_t k0 = int64_t(first + u) * 32 + q * 8;
          const bool in = first + u < u1 && k0 < p.x_k;
          a0[u] = in ? load_16(r0 + k0 * 2) : none;
          a1[u] = in ? load_16(r1 + k0 * 2) : none;
#pragma unroll
          for (int e = 0; e < kNt; ++e) {
            const int t = 8 * e + g;
            v[u][e] = in && t < tokens ? load_16(p.x + int64_t(t0 + t) * p.x_rs + k0 * 2) : none;
          }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
#pragma unroll
          for (int e = 0; e < kNt; ++e) {
            mma16<T>(acc[e], a0[u].x, a1[u].x, a0[u].y, a1[u].y, v[u][e].x, v[u][e].y);
            mma16<T>(acc[e], a0[u].z, a1[u].z, a0[u].w, a1[u].w, v[u][e].z, v[u][e].w);
          }
      }
#pragma unroll
      for (int e = 0; e < kNt; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = 16 * m + g + (i >> 1) * 8, t = 8 * e + 2 * q + (i & 1);
          if (row < p.E && t < tokens) part[(slice * tokens + t) * p.E + row] = acc[e][i];
        }
    }
  }
  float* const inbox = part + slices * chunk * p.E;
  const int own = (tokens + kRouterBlocks - 1) / kRouterBlocks * p.E;  // scores from one block
  __syncthreads();
  cluster_wait();  // every block of the cluster is there
  for (int i = threadIdx.x; i < tokens * p.E; i += kRouterWarps * 32) {
    const int t = i / p.E, e = i - t * p.E;
    float v = part[i];
    for (int o = 1; o < slices; ++o) v += part[o * tokens * p.E + i];
    store_cluster(cluster_map_shared(smem_u32(inbox + rank * own + t / kRouterBlocks * p.E + e), t % kRouterBlocks), v);
  }
  cluster_sync_all();
  for (int t = rank + kRouterBlocks * warp; t < tokens; t += kRouterBlocks * kRouterWarps) {
    // the token's scores, whole: the first of each lane's in registers, the others back in memory
    const float* const from = inbox + t / kRouterBlocks * p.E;
    uint32_t* const row = reinterpret_cast<uint32_t*>(inbox + t / kRouterBlocks * p.E);
    uint32_t key[4] = {}, top = 0;
    for (int e = lane, i = 0; e < p.E; e += 32, ++i) {
      float sum = 0.0f;
#pragma unroll
      for (int r = 0; r < kRouterBlocks; ++r) sum += from[r * own + e];
      const uint32_t k = key_of(sum);
      top = max(top, k);
#pragma unroll
      for (int j = 0; j < 4; ++j) key[j] = i == j ? k : key[j];
      if (i >= 4) row[e] = k;
    }
    const float largest = score_of(__reduce_max_sync(0xffffffffu, top));
    float sum = 0.0f;
    if (!p.normalize) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (key[i]) sum += expf(score_of(key[i]) - largest);
      for (int e = lane + 128; e < p.E; e += 32) sum += expf(score_of(row[e]) - largest);
    }
    // The largest k times; of equal ones the lowest number, which leaves the others behind.
    float mine = 0.0f;  // lane j: the j-th choice's score
    int id = 0;
    for (int j = 0; j < p.k; ++j) {
      uint32_t best = max(max(key[0], key[1]), max(key[2], key[3]));
      for (int e = lane + 128; e < p.E; e += 32) best = max(best, row[e]);
      best = __reduce_max_sync(0xffffffffu, best);
      uint32_t first = ~0u;
      for (int e = lane + 128; e < p.E && first == ~0u; e += 32) first = row[e] == best ? e : ~0u;
#pragma unroll
      for (int i = 3; i >= 0; --i) first = key[i] == best ? 32 * i + lane : first;
      const uint32_t e = __reduce_min_sync(0xffffffffu, first);
      if (first == e) {  // this lane's: gone
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = int(e) == 32 * i + lane ? 0 : key[i];
        if (e >= 128) row[e] = 0;
      }
      if (lane == j) mine = score_of(best), id = int(e);
    }
    if (p.normalize) sum = lane < p.k ? expf(mine - largest) : 0.0f;
    sum = warp_sum(sum);
    if (lane < p.k) {
      p.ids[int64_t(t0 + t) * p.ids_rs + lane * p.ids_cs] = id;
      p.weights[int64_t(t0 + t) * p.weights_rs + lane * p.weights_cs] = __fdiv_rn(expf(mine - largest), sum);
    }
  }
}

// ---- who goes where --------------------------------------------------------------------------------
// Of the tokens of a launch, in shared memory: the pairs (token, choice) in the order of experts, of an expert
// ascending by token, in groups of up to `most` of one expert.  An expert that a token names twice counts once, with
// both weights; numbers that are no expert's count for nothing.
struct Routes {
  uint64_t* tokens;   // [E]: bit t
  float* weight;      // [pairs], as `pairs` (down kernel)
  uint16_t *first_of;  // [E]
  uint16_t* pairs;    // [pairs]: t k + j
  uint16_t *expert, *first;  // [groups]
  uint8_t* count;     // [groups]
  uint8_t* token;     // [pairs], as `pairs`: t
  int groups;
};
constexpr __host__ __device__ int most_groups(int E, int pairs, int most) { return (E < pairs ? E : pairs) + pairs / most; }
constexpr int routes_bytes(int E, int pairs, int most, bool weights) {
  return E * 10 + pairs * (weights ? 13 : 5) + most_groups(E, pairs, most) * 5 + 16;
}

template <bool kWeights>
__device__ __forceinline__ Routes routes_of(const MoeParams& p, uint8_t* smem, int* scratch, int most) {
  const int E = p.E, pairs = p.T * p.k, tid = threadIdx.x, nt = kWarps * 32;
  Routes r;
  r.tokens = reinterpret_cast<uint64_t*>(smem);
  r.weight = reinterpret_cast<float*>(r.tokens + E);
  float* const given = r.weight + (kWeights ? pairs : 0);  // [pairs]: the weights as they are given
  int16_t* const ids = reinterpret_cast<int16_t*>(given + (kWeights ? pairs : 0));  // [pairs]: the experts, -1: none
  r.first_of = reinterpret_cast<uint16_t*>(ids + pairs);
  r.pairs = r.first_of + E;
  r.expert = r.pairs + pairs;
  r.first = r.expert + most_groups(E, pairs, most);
  r.count = reinterpret_cast<uint8_t*>(r.first + most_groups(E, pairs, most));
  r.token = r.count + most_groups(E, pairs, most);
  auto id_of = [&](int t, int j) { return __ldg(p.ids + t * p.ids_rs + j * p.ids_cs); };
  if (pairs <= 32) {  // one warp, a lane a pair: a kernel a microsecond and a half shorter than the general way
    if (tid < 32) {
      const uint32_t whole = 0xffffffffu;
      const int t = tid / p.k, id = tid < pairs ? id_of(t, tid - t * p.k) : -1;
      const bool valid = id >= 0 && id < E;
      const int key = valid ? id * kTokens + t : -1 - tid;
      const uint32_t same = __match_any_sync(whole, key);
      const bool counts = valid && __ffs(int(same)) - 1 == tid;
      float w = 0.0f;
      if (kWeights) {
        const float own = valid ? __ldg(p.weights + t * p.weights_rs + (tid - t * p.k) * p.weights_cs) : 0.0f;
        for (int j = 0; j < pairs; ++j) {
          const float v = __shfl_sync(whole, own, j);
          if (same >> j & 1) w += v;
        }
      }
      // places: pairs in front, of the same expert (`in`) and of others; one token's experts stay in their order
      const uint32_t real = __ballot_sync(whole, counts), mates = __match_any_sync(whole, counts ? id : -1 - tid);
      int at = __popc(real & ((1u << tid) - 1)), in = 0, group = at;
      if (p.T > 1) {
        at = 0;
        for (int j = 0; j < pairs; ++j) {
          const int other = __shfl_sync(whole, key, j);
          const bool front = (real >> j & 1) && other < key;
          at += front;
          in += front && (mates >> j & 1);
        }
      }
      const bool starts = counts && in % most == 0;
      const uint32_t heads = __ballot_sync(whole, starts);
      if (p.T > 1) {
        group = 0;
        for (int j = 0; j < pairs; ++j) {
          const int other = __shfl_sync(whole, at, j);
          group += (heads >> j & 1) && other < at;
        }
      }
      if (counts) {
        r.pairs[at] = uint16_t(tid);
        r.token[at] = uint8_t(t);
        if (kWeights) r.weight[at] = w;
      }
      if (starts) {
        r.expert[group] = uint16_t(id);
        r.first[group] = uint16_t(at);
        r.count[group] = uint8_t(min(most, __popc(mates) - in));
      }
      if (tid == 0) scratch[0] = __popc(heads);
    }
    __syncthreads();
    r.groups = scratch[0];
    return r;
  }
  for (int e = tid; e < E; e += nt) r.tokens[e] = 0;
  __syncthreads();
  for (int i = tid; i < pairs; i += nt) {
    const int t = i / p.k, e = id_of(t, i - t * p.k);
    if (kWeights) given[i] = __ldg(p.weights + t * p.weights_rs + (i - t * p.k) * p.weights_cs);
    ids[i] = int16_t(e >= 0 && e < E ? e : -1);
    if (e >= 0 && e < E) atomicOr(reinterpret_cast<unsigned long long*>(r.tokens + e), 1ull << t);
  }
  __syncthreads();
  // groups and pairs in front of each expert's: at most 1024 experts, 4 a thread
  int n[4], groups = 0, entries = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = tid * 4 + i;
    n[i] = e < E ? __popcll(r.tokens[e]) : 0;
    groups += (n[i] + most - 1) / most;
    entries += n[i];
  }
  const int both = groups | entries << 16;  // (at most 1536 and 2048)
  int incl = both;
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
  r.groups = total & 0xffff;
  int at = base & 0xffff, first = base >> 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = tid * 4 + i;
    if (n[i]) r.first_of[e] = uint16_t(first);
    for (int c = 0; c < n[i]; c += most, ++at) {
      r.expert[at] = uint16_t(e);
      r.first[at] = uint16_t(first + c);
      r.count[at] = uint8_t(min(most, n[i] - c));
    }
    first += n[i];
  }
  __syncthreads();
  for (int i = tid; i < pairs; i += nt) {
    const int t = i / p.k, j = i - t * p.k, e = ids[i];
    if (e < 0) continue;
    bool again = false;
    float w = kWeights ? given[i] : 0.0f;
    for (int o = 0; o < p.k; ++o) {
      if (o == j || ids[t * p.k + o] != e) continue;
      again |= o < j;
      if (kWeights) w += given[t * p.k + o];
    }
    if (again) continue;
    const int to = r.first_of[e] + __popcll(r.tokens[e] & ((1ull << t) - 1));
    r.pairs[to] = uint16_t(i);
    r.token[to] = uint8_t(t);
    if (kWeights) r.weight[to] = w;
  }
  __syncthreads();
  return r;
}

// ---- weights and tokens through a ring ---------------------------------------------------------------
// A unit is segments of 128 bytes: 16 of weights' rows, then a column each.  Segments of odd number have their halves
// swapped, so that the 16-byte words that eight lanes read together lie in different banks.
__device__ __forceinline__ uint32_t place(int segment, int byte) { return segment * 128 + (byte ^ ((segment & 1) << 6)); }

// 16 bytes, of which the first n are from memory and the others zeros, to shared memory, not waited for.
__device__ __forceinline__ void copy_piece(uint32_t to, const char* from, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
}
// Copies 16 bytes that every lane names of 4 rows (or columns) each, 128 bytes of 4 neighbouring rows an instruction;
// lane l's go to the word l % 8 of the rows l / 8, l / 8 + 4, ... of those from `segment` on.  Of columns, the first `count`.
template <int kEach>
__device__ __forceinline__ void copy_16(uint32_t to, int segment, int lane, const char* const (&from)[kEach], uint32_t at, bool there,
                                        int count) {
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (i * 4 + (lane >> 3) < count) copy_piece(to + place(segment + i * 4 + (lane >> 3), (lane & 7) * 16), from[i] + at, there ? 16 : 0);
}
// The weights where a row's elements lie step(s) apart: segment s is 64 elements from at(s), of which the first `left`
// are there and the others zeros.
template <typename At, typename Step>
__device__ __forceinline__ void copy_elements(uint8_t* ring, int lane, int left, At at, Step step) {
  for (int seg = 0; seg < 16; ++seg) {
    const uint16_t* from = reinterpret_cast<const uint16_t*>(at(seg));
    const int64_t cs = step(seg);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int e = i * 32 + lane;
      *reinterpret_cast<uint16_t*>(ring + place(seg, e * 2)) = e < left ? __ldg(from + e * cs) : uint16_t(0);
    }
  }
}
// The weights where rows begin at any multiple of 2 bytes: pieces of 16 bytes from the multiple of 16 that they begin
// at or behind, so that a row lies up to 14 bytes behind its segment's start and ends in a ninth piece (`kNinths`).  (That
// multiple lies in the row's allocation, which begins at one itself; behind a row's end nothing is read.)
constexpr int kNinths = 2048;  // where the ninth pieces lie in a unit: behind the weights
struct OddRows {
  // of rows l / 8, l / 8 + 4, ... (l: the lane) the lane's piece of eight, of row l the ninth; and the bytes from there to
  // the row's end
  const char *at[4], *ninth;
  uint32_t left[4], ninth_left;
  template <typename Row>
  __device__ __forceinline__ void aim(int lane, uint32_t row_bytes, Row row_of) {
    auto piece = [&](const char* row, int byte, uint32_t* left) {
      const uint32_t behind = uint32_t(reinterpret_cast<uintptr_t>(row)) & 15u;
      *left = row_bytes + behind - byte;  // (may lie behind the end: below zero)
      return row - behind + byte;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) at[i] = piece(row_of(i * 4 + (lane >> 3)), (lane & 7) * 16, &left[i]);
    ninth = piece(row_of(lane & 15), 128, &ninth_left);
  }
  // The unit that begins `from` bytes behind the rows' first elements.
  __device__ __forceinline__ void copy(uint8_t* unit, int lane, uint32_t from) const {
    auto put = [&](uint32_t to, const char* p, uint32_t left) {
      const uint32_t bytes = uint32_t(max(0, min(16, int(left - from))));
      copy_piece(to, p + (bytes ? int64_t(from) : 0), bytes);
    };
    const uint32_t to = smem_u32(unit);
#pragma unroll
    for (int i = 0; i < 4; ++i) put(to + place(i * 4 + (lane >> 3), (lane & 7) * 16), at[i], left[i]);
    if (lane < 16) put(to + kNinths + lane * 16, ninth, ninth_left);
  }
};
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kStages>
__device__ __forceinline__ void wait_for_unit() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
  __syncwarp();
}
__device__ __forceinline__ uint4 words_at(const uint8_t* unit, int segment, int byte) {
  return *reinterpret_cast<const uint4*>(unit + place(segment, byte));
}
// The same of weights that OddRows brought; behind: bytes from the segment's start to the row.
__device__ __forceinline__ uint4 odd_words_at(const uint8_t* unit, int segment, int byte, uint32_t behind) {
  const uint4 a = words_at(unit, segment, byte);
  const uint4 b = *reinterpret_cast<const uint4*>(byte == 112 ? unit + kNinths + segment * 16 : unit + place(segment, byte + 16));
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  const bool two = behind & 8, one = behind & 4;
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = two ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = one ? w[i + 1] : w[i];
  const uint32_t bits = (behind & 2) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}
__device__ __forceinline__ uint32_t behind_16(const char* row) { return uint32_t(reinterpret_cast<uintptr_t>(row)) & 15u; }
__device__ __forceinline__ int left_of(int64_t length, int64_t from) { return int(min(max(length - from, int64_t(0)), int64_t(64))); }

// ---- gate and up ------------------------------------------------------------------------------------
// Team b of kTeam warps (a block or, where channels are few, less) takes the items b, b + teams, ... of (group, 8 hidden
// channels), which its warps share in units of 64 channels.  Rows 0 to 7 of a tile are the gate's, rows 8 to 15 the up
// projection's.
template <typename T, int kNt, bool kOdd>
struct GateUp {
  static constexpr int kFirst = kOdd ? 18 : 16;  // the columns' first segment
  static constexpr int kStages = kNt == 1 ? 4 : 3, kUnitBytes = kFirst * 128 + kNt * 1024, kColumns = 8 * kNt;
  static constexpr int kRing = kWarps * kStages * kUnitBytes, kSmem = kRing + kWarps * kNt * 512;
};
template <typename T, int kNt, int kTeam, bool kOdd>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_moe_gate_up_kernel(const MoeParams p) {
  using S = GateUp<T, kNt, kOdd>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int scratch[kWarps];
  float(*const sums)[128] = reinterpret_cast<float(*)[128]>(smem + S::kRing);  // [kNt * kWarps]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  uint8_t* const ring = smem + warp * (S::kStages * S::kUnitBytes);
  start_in_order();
  const Routes r = routes_of<false>(p, smem + S::kSmem, scratch, S::kColumns);
  const int tiles = int((p.F + 7) / 8);
  constexpr int kTeams = kWarps / kTeam;
  // (teams of a block are gridDim.x apart, so that a last round spreads over the SMs)
  const int team = int(blockIdx.x) + warp / kTeam * int(gridDim.x), member = warp % kTeam, thread = threadIdx.x % (kTeam * 32);
  auto team_sync = [&]() {
    if constexpr (kTeams == 1) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / kTeam), "n"(kTeam * 32) : "memory");
  };
  const int units = int((p.D + 63) / 64), per = (units + kTeam - 1) / kTeam, u0 = member * per;
  const int64_t items = int64_t(r.groups) * tiles, stride = int64_t(gridDim.x) * kTeams;
  const int64_t mine = team < items ? (items - 1 - team) / stride + 1 : 0;

  // (an item's group and tile, kept without divisions)
  const int step_group = int(stride / tiles), step_tile = int(stride % tiles);
  int lgroup = team / tiles, ltile = team % tiles, lu = 0, lcount = 0;
  const char *rows[4], *columns[2 * kNt];  // of the item: what this lane copies of
  auto row_at = [&](int64_t e, int tile, int seg) {
    const int64_t f = min(int64_t(tile) * 8 + (seg & 7), p.F - 1);
    return seg < 8 ? p.w_gate + (e * p.gate_es + f * p.gate_rs) * 2 : p.w_up + (e * p.up_es + f * p.up_rs) * 2;
  };
  OddRows odd;
  auto row_of = [&](int64_t e, int seg) { return row_at(e, ltile, seg); };
  auto aim = [&]() {
    if (lgroup >= r.groups) return;
    const int64_t e = r.expert[lgroup];
    const int first = r.first[lgroup];
    lcount = r.count[lgroup];
    if constexpr (kOdd) odd.aim(lane, uint32_t(p.D) * 2, [&](int seg) { return row_of(e, seg); });
    if (!kOdd && p.piece_in == 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) rows[i] = row_of(e, i * 4 + (lane >> 3));
    }
#pragma unroll
    for (int i = 0; i < 2 * kNt; ++i) columns[i] = p.x + int64_t(r.token[first + min(i * 4 + (lane >> 3), lcount - 1)]) * p.x_rs;
  };
  const uint32_t row_bytes = uint32_t(p.D) * 2, column_bytes = uint32_t(p.x_k) * 2;
  auto load = [&](int stage) {
    const int unit = u0 + lu;
    if (lgroup < r.groups && unit < units) {
      uint8_t* const to = ring + stage * S::kUnitBytes;
      const uint32_t at = uint32_t(unit) * 128 + (lane & 7) * 16;
      if constexpr (kOdd) {
        odd.copy(to, lane, uint32_t(unit) * 128);
      } else if (p.piece_in == 16) {
        copy_16(smem_u32(to), 0, lane, rows, at < row_bytes ? at : 0, at < row_bytes, 16);
      } else {
        const int64_t e = r.expert[lgroup], k0 = int64_t(unit) * 64;
        copy_elements(to, lane, left_of(p.D, k0), [&](int seg) { return row_of(e, seg) + k0 * (seg < 8 ? p.gate_cs : p.up_cs) * 2; },
                  [&](int seg) { return seg < 8 ? p.gate_cs : p.up_cs; });
      }
      copy_16(smem_u32(to), S::kFirst, lane, columns, at < column_bytes ? at : 0, at < column_bytes, lcount);
    }
    commit_copies();
    if (++lu == per) {
      lu = 0;
      ltile += step_tile;
      lgroup += step_group;
      if (ltile >= tiles) ltile -= tiles, ++lgroup;
      aim();
    }
  };
  aim();
  for (int i = 0; i < S::kStages; ++i) load(i);

  int group = team / tiles, tile = team % tiles, step = 0;
  float acc[kNt][4] = {};
  uint32_t behind[2] = {0, 0};  // of this lane's rows (kOdd)
  auto use = [&](int stage) {
    const int count = r.count[group], unit = u0 + step;
    if (kOdd && step == 0) {
      const int64_t e = r.expert[group];
      behind[0] = behind_16(row_at(e, tile, g)), behind[1] = behind_16(row_at(e, tile, g + 8));
    }
    wait_for_unit<S::kStages>();
    if (unit < units) {
      const uint8_t* from = ring + stage * S::kUnitBytes;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = i * 64 + q * 16;
        const uint4 a0 = kOdd ? odd_words_at(from, g, at, behind[0]) : words_at(from, g, at);
        const uint4 a1 = kOdd ? odd_words_at(from, g + 8, at, behind[1]) : words_at(from, g + 8, at);
#pragma unroll
        for (int e = 0; e < kNt; ++e) {
          if (8 * e >= count) break;
          const uint4 v = words_at(from, S::kFirst + 8 * e + g, at);  // (columns behind the last: whatever lies there)
          mma16<T>(acc[e], a0.x, a1.x, a0.y, a1.y, v.x, v.y);
          mma16<T>(acc[e], a0.z, a1.z, a0.w, a1.w, v.z, v.w);
        }
      }
    }
    __syncwarp();
    if (++step < per) return;
    step = 0;
    team_sync();  // the sums before have been read
#pragma unroll
    for (int e = 0; e < kNt; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sums[e * kWarps + warp][i * 32 + lane] = acc[e][i];
        acc[e][i] = 0.0f;
      }
    team_sync();
    for (int i = thread; i < 8 * count; i += kTeam * 32) {
      const int f = i & 7, c = i >> 3, at = (c & 1) * 32 + f * 4 + ((c & 7) >> 1);
      const float(*part)[128] = sums + (c >> 3) * kWarps + (warp - member);
      float a[1] = {0.0f}, u[1] = {0.0f};
#pragma unroll
      for (int w = 0; w < kTeam; ++w) {
        a[0] += part[w][at];
        u[0] += part[w][at + 64];
      }
      gate(p.act, a, u);
      const int64_t channel = int64_t(tile) * 8 + f, to = int64_t(r.pairs[r.first[group] + c]) * p.h_rs + channel;
      if (channel >= p.F) a[0] = 0.0f;  // the rest of the row's last 16 bytes
      const T hi = from_f32<T>(a[0]);
      reinterpret_cast<T*>(p.h)[to] = hi;
      // (what overflows has no second part)
      reinterpret_cast<T*>(p.h_lo)[to] = from_f32<T>(isfinite(to_f32(hi)) ? a[0] - to_f32(hi) : 0.0f);
    }
    tile += step_tile;
    group += step_group;
    if (tile >= tiles) tile -= tiles, ++group;
  };
  const int64_t total = mine * per;
  int stage = 0;
  for (int64_t it = 0; it < total; ++it) {
    use(stage);
    load(stage);
    if (++stage == S::kStages) stage = 0;
  }
}

// ---- down -------------------------------------------------------------------------------------------
// Cluster c of `parts` blocks takes the tiles c, c + clusters, ... of 16 channels, each through all groups; the (group,
// 64 hidden channels) of a tile are dealt evenly to the cluster's warps, in order.  Columns are a group's tokens, the
// first parts of h in kNt tiles of them and the second parts in kNt more.  Each warp adds its groups' sums, times their
// weights, to sums of its own [token][16] in shared memory; those of the warps are added up in order, sent to the block
// that writes them (block r of n has the r-th of n neighbours), and there the blocks' in order.
template <typename T, int kNt, bool kOdd>
struct Down {
  static constexpr int kFirst = kOdd ? 18 : 16;  // the columns' first segment
  static constexpr int kUnitBytes = kFirst * 128 + kNt * 2048, kTokens = 8 * kNt;
  static int ring(int stages) { return kWarps * stages * kUnitBytes; }
};
// What the blocks of a cluster send one of them of a tile, in multiples of 8 bytes.  (A tile that is shared is its
// cluster's only one: parts of 2 and more are chosen where the device has a cluster for each tile.)
constexpr __host__ __device__ int box_bytes(int T, int parts) { return parts == 1 ? 0 : ((T * 16 + parts - 1) / parts * parts + 1) / 2 * 8; }
template <typename T, int kNt, int kStages, bool kOdd>
__global__ void __launch_bounds__(kWarps * 32, 2) cconv_moe_down_kernel(const MoeParams p, const int parts) {
  using S = Down<T, kNt, kOdd>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int scratch[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  uint8_t* const ring = smem + warp * (kStages * S::kUnitBytes);
  float* const all = reinterpret_cast<float*>(smem + kWarps * kStages * S::kUnitBytes);  // [kWarps][T][16]
  float* const mine = all + warp * p.T * 16;
  const int tiles = int((p.D + 15) / 16), clusters = int(gridDim.x) / parts;
  const int rank = int(blockIdx.x) % parts, first_tile = int(blockIdx.x) / parts;
  const int units = int((p.F + 63) / 64);
  if (parts > 1) cluster_arrive();

  // Behind the gate and up kernel of the same call, which lets this one in only once everything before the call and the
  // router are complete, the choice and the weights are there already; h is waited for below.
  const Routes r = routes_of<true>(p, smem + kWarps * (kStages * S::kUnitBytes + p.T * 64) + box_bytes(p.T, parts), scratch, S::kTokens);
  const int64_t work = int64_t(r.groups) * units;
  const int64_t w0 = work * (rank * kWarps + warp) / (parts * kWarps), w1 = work * (rank * kWarps + warp + 1) / (parts * kWarps);
  const int each = int(w1 - w0), group0 = units ? int(w0 / units) : 0, unit0 = int(w0 - int64_t(group0) * units);

  // weights, and tokens once they are there
  int lt = first_tile, lgroup = group0, lunit = unit0, ln = 0, lcount = 0;
  const char *rows[4], *highs[2 * kNt], *lows[2 * kNt];  // of the tile and group: what this lane copies of
  const uint32_t row_bytes = uint32_t(p.F) * 2, column_bytes = uint32_t(p.h_rs) * 2;
  auto row_at = [&](int64_t e, int tile, int seg) {
    return p.w_down + (e * p.down_es + min(int64_t(tile) * 16 + seg, p.D - 1) * p.down_rs) * 2;
  };
  OddRows odd;
  auto row_of = [&](int64_t e, int seg) { return row_at(e, lt, seg); };
  auto aim = [&]() {
    if (lgroup >= r.groups) return;
    const int first = r.first[lgroup];
    lcount = r.count[lgroup];
    if constexpr (kOdd) odd.aim(lane, uint32_t(p.F) * 2, [&](int seg) { return row_of(r.expert[lgroup], seg); });
    if (!kOdd && p.piece_out == 16) {
      const int64_t e = r.expert[lgroup];
#pragma unroll
      for (int i = 0; i < 4; ++i) rows[i] = row_of(e, i * 4 + (lane >> 3));
    }
#pragma unroll
    for (int i = 0; i < 2 * kNt; ++i) {
      const int64_t h = int64_t(r.pairs[first + min(i * 4 + (lane >> 3), lcount - 1)]) * column_bytes;
      highs[i] = p.h + h;
      lows[i] = p.h_lo + h;
    }
  };
  auto load_weights = [&](int stage) {
    uint8_t* const to = ring + stage * S::kUnitBytes;
    if constexpr (kOdd) {
      odd.copy(to, lane, uint32_t(lunit) * 128);
    } else if (p.piece_out == 16) {
      const uint32_t at = uint32_t(lunit) * 128 + (lane & 7) * 16;
      copy_16(smem_u32(to), 0, lane, rows, at < row_bytes ? at : 0, at < row_bytes, 16);
    } else {
      const int64_t e = r.expert[lgroup], k0 = int64_t(lunit) * 64;
      copy_elements(to, lane, left_of(p.F, k0), [&](int seg) { return row_of(e, seg) + k0 * p.down_cs * 2; },
                [&](int) { return p.down_cs; });
    }
  };
  auto load_tokens = [&](int stage) {
    const uint32_t to = smem_u32(ring + stage * S::kUnitBytes), at = uint32_t(lunit) * 128 + (lane & 7) * 16;
    copy_16(to, S::kFirst, lane, highs, at < column_bytes ? at : 0, at < column_bytes, lcount);
    copy_16(to, S::kFirst + S::kTokens, lane, lows, at < column_bytes ? at : 0, at < column_bytes, lcount);
  };
  auto next = [&]() {
    if (++ln == each) {
      ln = 0;
      lgroup = group0;
      lunit = unit0;
      lt += clusters;
      aim();
    } else if (++lunit == units) {
      lunit = 0;
      ++lgroup;
      aim();
    }
  };
  auto fill = [&](auto load, auto commit) {
    lt = first_tile, lgroup = group0, lunit = unit0, ln = 0;
    aim();
    for (int i = 0; i < kStages; ++i) {
      if (each && lt < tiles) load(i);
      commit();
      next();
    }
  };
  fill(load_weights, [] {});
  start_in_order();
  fill(load_tokens, [] { commit_copies(); });  // (the first takes in the weights of all stages)
  if (parts > 1) cluster_wait();  // every block of the cluster is there
  const int outputs = p.T * 16, share = (outputs + parts - 1) / parts;
  float* const box = all + kWarps * outputs;  // [parts][share]
  auto put_out = [&](int tile, int i, float v) {
    const int64_t channel = int64_t(tile) * 16 + (i & 15);
    if (channel < p.D) static_cast<T*>(const_cast<void*>(p.out.p))[(i >> 4) * p.out.rs + channel * p.out.cs] = from_f32<T>(v);
  };
  int stage = 0;
  for (int tile = first_tile; tile < tiles; tile += clusters) {
    for (int i = lane; i < p.T * 16; i += 32) mine[i] = 0.0f;
    __syncwarp();
    float d[2 * kNt][4] = {};
    int group = group0, unit = unit0;
    uint32_t behind[2] = {0, 0};  // of this lane's rows (kOdd)
    for (int n = 0; n < each; ++n) {
      const int count = r.count[group];
      if (kOdd && (n == 0 || unit == 0)) {
        const int64_t e = r.expert[group];
        behind[0] = behind_16(row_at(e, tile, g)), behind[1] = behind_16(row_at(e, tile, g + 8));
      }
      wait_for_unit<kStages>();
      const uint8_t* from = ring + stage * S::kUnitBytes;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = i * 64 + q * 16;
        const uint4 a0 = kOdd ? odd_words_at(from, g, at, behind[0]) : words_at(from, g, at);
        const uint4 a1 = kOdd ? odd_words_at(from, g + 8, at, behind[1]) : words_at(from, g + 8, at);
#pragma unroll
        for (int e = 0; e < 2 * kNt; ++e) {
          if (8 * (e % kNt) >= count) continue;
          const uint4 v = words_at(from, S::kFirst + 8 * e + g, at);
          mma16<T>(d[e], a0.x, a1.x, a0.y, a1.y, v.x, v.y);
          mma16<T>(d[e], a0.z, a1.z, a0.w, a1.w, v.z, v.w);
        }
      }
      __syncwarp();
      if (lt < tiles) {
        load_weights(stage);
        load_tokens(stage);
      }
      commit_copies();
      next();
      if (++stage == kStages) stage = 0;
      if (++unit == units || n + 1 == each) {
        // the group's share: this lane's columns are tokens 2q and 2q + 1 of eight
        const int first = r.first[group];
#pragma unroll
        for (int e = 0; e < kNt; ++e)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int column = 8 * e + 2 * q + c;
            if (column < count) {
              const float w = r.weight[first + column];
              float* to = mine + r.token[first + column] * 16 + g;
              to[0] += w * (d[e][c] + d[kNt + e][c]);
              to[8] += w * (d[e][2 + c] + d[kNt + e][2 + c]);
            }
            d[e][c] = d[kNt + e][c] = d[e][2 + c] = d[kNt + e][2 + c] = 0.0f;
          }
        __syncwarp();
        unit = 0;
        ++group;
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < outputs; i += kWarps * 32) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) s += all[w * outputs + i];
      if (parts == 1) put_out(tile, i, s);
      else store_cluster(cluster_map_shared(smem_u32(box + rank * share + i / parts), i % parts), s);
    }
    if (parts == 1) {
      __syncthreads();
      continue;
    }
    cluster_sync_all();
    for (int i = threadIdx.x * parts + rank; i < outputs; i += parts * kWarps * 32) {
      float s = 0.0f;
      for (int b = 0; b < parts; ++b) s += box[b * share + i / parts];
      put_out(tile, i, s);
    }
  }
}

// ---- launches ---------------------------------------------------------------------------------------
constexpr int kMostShared = 200 * 1024;  // of a block here

template <typename T, int kNt>
cudaError_t launch_router(const MoeParams& p, int chunk, cudaStream_t s) {
  auto f = cconv_moe_router_kernel<T, kNt>;
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, kMostShared);
  if (e != cudaSuccess) return e;
  const int groups = int(cdiv64(p.E, 16)), slices = groups >= kRouterWarps ? 1 : kRouterWarps / groups;
  const dim3 grid(unsigned(cdiv64(p.T, chunk) * kRouterBlocks));
  const int64_t scores = int64_t(slices) * chunk + round_up64(chunk, kRouterBlocks);
  return launch(f, grid, kRouterWarps * 32, size_t(scores * p.E * 4), kRouterBlocks, s, p, chunk);
}
// Calls f(T(), columns of 8) for the call's type and at most 64 tokens.
template <typename F>
cudaError_t with_columns(int dtype, int64_t tokens, F f) {
  auto columns = [&](auto type) {
    if (tokens <= 8) return f(type, std::integral_constant<int, 1>());
    if (tokens <= 16) return f(type, std::integral_constant<int, 2>());
    if (tokens <= 32) return f(type, std::integral_constant<int, 4>());
    return f(type, std::integral_constant<int, 8>());
  };
  return dtype == CCONV_TYPE_BF16 ? columns(__nv_bfloat16()) : columns(__half());
}
// Tokens that choose together: as many as leave their scores room in shared memory.
int router_tokens(int64_t T, int64_t E) { return int(std::min<int64_t>(std::min<int64_t>(T, kTokens), std::max<int64_t>(8, 16384 / E))); }

template <typename T, int kNt, int kTeam, bool kOdd>
cudaError_t launch_gate_up_as(const MoeParams& p, int sms, cudaStream_t s) {
  using S = GateUp<T, kNt, kOdd>;
  auto f = cconv_moe_gate_up_kernel<T, kNt, kTeam, kOdd>;
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, kMostShared);
  if (e != cudaSuccess) return e;
  const int pairs = p.T * p.k;
  const int64_t most = cdiv64(most_groups(p.E, pairs, S::kColumns) * cdiv64(p.F, 8), kWarps / kTeam);
  return launch(f, dim3(unsigned(std::min<int64_t>(most, 2 * sms))), kWarps * 32,
                S::kSmem + routes_bytes(p.E, pairs, S::kColumns, false), 1, s, p);
}
constexpr int64_t kFewChannels = 768;  // 576 channels: 32.1 against 34.8 us with teams of 8, 1000: 27.1 against 26.6
template <typename T, int kNt>
cudaError_t launch_gate_up(const MoeParams& p, int sms, cudaStream_t s) {
  const bool few = p.D <= kFewChannels;
  if (p.piece_in == 2) return few ? launch_gate_up_as<T, kNt, 2, true>(p, sms, s) : launch_gate_up_as<T, kNt, 8, true>(p, sms, s);
  return few ? launch_gate_up_as<T, kNt, 2, false>(p, sms, s) : launch_gate_up_as<T, kNt, 8, false>(p, sms, s);
}
template <typename T, int kNt, int kStages, bool kOdd>
cudaError_t launch_down_odd(const MoeParams& p, int sms, cudaStream_t s) {
  using S = Down<T, kNt, kOdd>;
  auto f = cconv_moe_down_kernel<T, kNt, kStages, kOdd>;
  static bool ready[64] = {};
  const cudaError_t e = allow_smem(f, ready, kMostShared);
  if (e != cudaSuccess) return e;
  // blocks that share a tile, so that every SM has two
  const int64_t tiles = cdiv64(p.D, 16);
  const int parts = tiles * 2 > 2 * sms ? 1 : tiles * 4 > 2 * sms ? 2 : tiles * 8 > 2 * sms ? 4 : 8;
  const int64_t blocks = parts == 1 ? std::min<int64_t>(tiles, 2 * sms) : tiles * parts;
  return launch(f, dim3(unsigned(blocks)), kWarps * 32,
                S::ring(kStages) + kWarps * p.T * 64 + box_bytes(p.T, parts) + routes_bytes(p.E, p.T * p.k, S::kTokens, true), parts, s, p, parts);
}
template <typename T, int kNt, int kStages>
cudaError_t launch_down_as(const MoeParams& p, int sms, cudaStream_t s) {
  return p.piece_out == 2 ? launch_down_odd<T, kNt, kStages, true>(p, sms, s) : launch_down_odd<T, kNt, kStages, false>(p, sms, s);
}
template <typename T>
cudaError_t launch_layer(const MoeParams& p, int sms, cudaStream_t s) {
  // columns for 8 tokens of an expert, or for 16 where most have more than 8
  const bool many = int64_t(p.T) * p.k > 6 * int64_t(p.E) && p.T > 8;
  const cudaError_t e = many ? launch_gate_up<T, 2>(p, sms, s) : launch_gate_up<T, 1>(p, sms, s);
  if (e != cudaSuccess) return e;
  if (many) return launch_down_as<T, 2, 2>(p, sms, s);
  return p.T <= 16 ? launch_down_as<T, 1, 3>(p, sms, s) : launch_down_as<T, 1, 2>(p, sms, s);
}

// Bytes that rows of an expert's matrix begin at multiples of: 16 (and end there), 2, or 1: elements lie apart.
int piece_of(const cconv_matrix& m, int64_t expert_stride, int64_t rows, int64_t cols, int64_t experts) {
  if (m.col_stride != 1 && cols > 1) return 1;
  const uintptr_t lies = reinterpret_cast<uintptr_t>(m.data) | uintptr_t(rows > 1 ? m.row_stride * 2 : 0) |
                         uintptr_t(experts > 1 ? expert_stride * 2 : 0) | uintptr_t(cols * 2);
  return (lies & 15) == 0 ? 16 : 2;
}

void plan(Steps& st, const cconv_moe_args& a) {
  const int sms = st.sms();
  MoeParams p{};
  Padded padded;
  const Mat x = padded.readable(st, a.x, a.T, a.D, &p.x_k);
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
    const Mat router = padded.readable(st, a.router, a.E, a.D, &k);
    p.router = static_cast<const char*>(router.p);
    p.router_rs = router.rs * 2;
  }
  padded.add(st);
  if (a.router.data) {
    MoeParams r = p;
    r.T = int(a.T);
    st.add([=](cudaStream_t s) {
      const int chunk = router_tokens(r.T, r.E);
      return block_cuda_error(with_columns(r.dtype, chunk, [&](auto type, auto nt) {
        return launch_router<decltype(type), decltype(nt)::value>(r, chunk, s); }),
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
      return block_cuda_error(c.dtype == CCONV_TYPE_BF16 ? launch_layer<__nv_bfloat16>(c, sms, s) : launch_layer<__half>(c, sms, s),
                              "cconv_moe_forward");
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
