// Products of the feed-forward block on pairs of CTAs.
//
// C = A B^T over a 256 x block_n tile a pair: each CTA keeps 128 rows of A and half the rows of B in shared
// memory (64 elements of k a stage), one thread of the first CTA issues the MMAs of both (M = 256), and
// each CTA's accumulators (128 x block_n, fp32) lie in its own tensor memory, twice, so that a tile's
// epilogue runs beside the next tile's main loop.  A pair reads (256 + block_n) rows of k from L2 for
// 256 x block_n products, half of what two CTAs on tiles of their own would: at 128 x 256 a CTA draws 96
// bytes a clock, a pair of CTAs at 256 x 256 64 bytes a clock each, below what L2 delivers to an SM.
//
// A product with fewer tiles than pairs is cut along k: a cluster of 2 or 4 pairs shares a tile, each pair
// sums a part of k, and the pairs then exchange their accumulators through distributed shared memory, so
// that each finishes its own share of the columns (in the order of the parts: the result does not depend
// on who is first).  One launch, no table of partial sums in memory.
//
// Roles: warps 0 and 3 copy (TMA), warp 1 of the first CTA issues MMAs, warp 2 owns the tensor memory, warps
// 4-11 are the epilogue (two for each quarter of the lanes, half of the columns each).
//
// What bounds it: long products the tensor cores, under the power limit (8192 x 4096 x 8192, forward of the whole
// block, 1.65 PFLOP: 1.29 ms, 1.28 PFLOP/s at 1.3 to 1.4 GHz; backward 2.65 ms, 1.25 PFLOP/s).  Short ones
// what a launch costs before its first and after its last MMA (8 us with a round of tiles) and the latency of a
// stage: 64 to 256 tokens at 2048 x 8192 take 40 us forward, 8-bit 8192 x 4096 17 us.  The backward epilogue
// (dg, du and h from dh, g and u: 20 bytes an element) outlasts its tile's main loop up to k = 2048 (tensor cores
// busy 49 % at 4096 x 2048 x 8192, 73 % in the forward product).  8-bit sums are scaled at 800 clocks a block of
// 256 columns, where the MMAs take 512: 8192 x 8192 x 4096 295 to 300 us, 1.83 PFLOP/s (main loop alone 200 us
// under the power limit; 16 epilogue warps of 64 columns each: 338 us; loads of the next block's sums begun before
// this one's are added: 390 us).
#include <algorithm>
#include <cstdio>
#include <cstdlib>

#include "block.h"
#include "block_device.cuh"
#include "block_gemm.h"
#include "block_launch.h"
#include "pair_sm100.cuh"

namespace cconv {
namespace {

constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr uint32_t kABytes = 128 * 128;  // a stage of A in one CTA: 128 rows x 128 bytes of k
constexpr uint32_t kBoxBytes = 32 * 128; // a piece that an epilogue warp stages: 32 rows x 128 bytes
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kSmemMost = 232448;
constexpr uint32_t kBarrierBytes = 512;
constexpr int kMostStages = 16;

__device__ int g_block_status;

// A product of the launch, as the kernel sees it.
struct ProductParams {
  int tiles_m, tiles_n, first;  // first: tiles of the products before it
  int kb_total, kb_seg, kb_part;  // k blocks: all, of the first segment, of a pair's part
  int block_n;
  uint32_t a_bytes, b_bytes;    // what a stage brings of A and B to one CTA
  uint32_t one_sided;           // the rows of A are all the first CTA's
  uint32_t a_kmajor, b_kmajor;
  uint32_t a_step, b_step;      // descriptor step of 16 elements of k (16-byte units)
  uint32_t idesc;
  uint64_t a_desc, b_desc;
  int64_t M, N;
};
template <int kProducts>
struct PairParams {
  ProductParams of[kProducts];
  int count, tiles, splits, stages;
  uint32_t a_stage, stage_bytes; // room of a stage's A; of the whole stage
  uint32_t pieces;              // staged by an epilogue warp
  int paired, act, save;
  // cut: where results go and come from (in elements)
  char* out[3];
  int64_t out_rs[3], out_cs[3];
  const char* in[2];
  int64_t in_rs[2];
  // 8-bit: scale of row r (of 128 rows of B) and k block kb
  const float *row_scale, *col_scale;
  int64_t row_rs, row_ks, col_rs, col_ks;
  int* status;
  uint64_t limit_ns;
};
struct ProductMaps {
  CUtensorMap a[2], b[2], out;
};
template <int kProducts>
struct PairMaps {
  ProductMaps of[kProducts];
};
template <>
struct PairMaps<1> {
  ProductMaps of[1];
  CUtensorMap out1, out2, in[2];
};
template <int kEpi>
constexpr int kProductsOf = kEpi == kStore ? kMostProducts : 1;

// Tile t of the launch: product, row and column of tiles.  Tiles run down groups of 8 rows of tiles, so that
// the pairs at work at one time read few different rows of A and B.
struct Tile {
  int of, m, n;
};
template <int kProducts>
__device__ __forceinline__ Tile tile_of(const PairParams<kProducts>& p, int t) {
  Tile r;
  r.of = 0;
  if (kProducts > 1) {
    while (r.of + 1 < p.count && t >= p.of[r.of + 1].first) ++r.of;
    t -= p.of[r.of].first;
  }
  const int tiles_n = p.of[r.of].tiles_n, tiles_m = p.of[r.of].tiles_m;
  const int group = 8 * tiles_n;
  const int first = t / group * 8;
  const int rows = min(8, tiles_m - first);
  t %= group;
  r.m = first + t % rows;
  r.n = t / rows;
  return r;
}

// Waits for this thread's loads from tensor memory; what they brought is not used before.
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                 "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
                 "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
                 "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_ld_hold(uint32_t (&v)[32]) {  // as after a wait that has been made
  asm volatile("" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                 "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
                 "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
                 "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]));
}
__device__ __forceinline__ void load_sums(uint32_t taddr, float (&f)[32]) {
  uint32_t v[32];
  tmem_ld_32x32b_x32(taddr, v);
  tmem_ld_wait(v);
#pragma unroll
  for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
}

// Eight columns (cut along k, where code that a launch fetches cold and runs once had better be short).
__device__ __forceinline__ void load_sums8(uint32_t taddr, float (&f)[8]) {
  uint32_t v[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(taddr)
               : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7])
               :
               : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[i]);
}

// 16-byte chunk c of row r of a piece staged with 128-byte swizzle.
__device__ __forceinline__ uint32_t chunk_at(uint32_t base, int r, int c) {
  return base + r * 128 + ((c ^ (r & 7)) << 4);
}
template <typename T>
__device__ __forceinline__ void stage32(uint32_t base, int r, int c0, const float (&f)[32]) {
#pragma unroll
  for (int c = 0; c < 4; ++c)
    st_shared_v4(chunk_at(base, r, c0 + c), pack2<T>(f[8 * c], f[8 * c + 1]), pack2<T>(f[8 * c + 2], f[8 * c + 3]),
                 pack2<T>(f[8 * c + 4], f[8 * c + 5]), pack2<T>(f[8 * c + 6], f[8 * c + 7]));
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
}
template <typename T>
__device__ __forceinline__ void unpack8(const uint4& w, float (&f)[8]) {
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = unpack2<T>(a[i]);
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
}
template <typename T>
__device__ __forceinline__ void unstage32(uint32_t base, int r, int c0, float (&f)[32]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint4 w;
    ld_shared_v4(chunk_at(base, r, c0 + c), w.x, w.y, w.z, w.w);
    float v[8];
    unpack8<T>(w, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[8 * c + i] = v[i];
  }
}

// Pieces that an epilogue warp stages.
int pieces_of(const Launch& l) {
  if (l.cut()) return 0;
  return l.epilogue == kStore ? 2 : l.epilogue == kScaled || (l.epilogue == kGated && !l.save) ? 1 : 3;
}
// Scales of 8-bit rows that an epilogue warp keeps: 16 blocks of k of its 32 rows and of its columns
// (row 32), the 16 in use and the next 16; a pitch of 17 words keeps the lanes on different banks.
constexpr uint32_t kScaleBytes = 33 * 17 * 4;
uint32_t scale_bytes(int epi) { return epi == kScaled ? 2 * kEpilogueWarps * kScaleBytes : 0; }
// Rows of A that a stage brings to a CTA: 128, or fewer where the product has fewer (the tensor cores then
// read what lies behind them for rows that nobody stores).  A stage of a few tokens is mostly weights, so that
// more of those are on their way.
int a_rows_of(const Product& p) {
  const int least = p.a[0].kmajor ? 16 : 64;
  int rows = 128;
  while (rows > least && p.M <= rows / 2) rows /= 2;
  return rows;
}
int stages_of(const Launch& l, uint32_t a_bytes, uint32_t b_bytes) {
  const uint32_t other = 1024 + kBarrierBytes + kEpilogueWarps * pieces_of(l) * kBoxBytes + scale_bytes(l.epilogue) + kABytes - a_bytes;
  return std::min(kMostStages, int((kSmemMost - other) / (a_bytes + b_bytes)));
}

__device__ __forceinline__ void cp_async4(uint32_t to, const float* from, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ float ld_shared_f32(uint32_t at) {
  float f;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(at) : "memory");
  return f;
}
__device__ __forceinline__ void stage_f32(uint32_t base, int r, const float* f) {
#pragma unroll
  for (int c = 0; c < 8; ++c)
    st_shared_v4(chunk_at(base, r, c), __float_as_uint(f[4 * c]), __float_as_uint(f[4 * c + 1]),
                 __float_as_uint(f[4 * c + 2]), __float_as_uint(f[4 * c + 3]));
}

// A bounded wait whose outcome is the same in all lanes, so that a warp leaves as a whole.
__device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int code,
                                         uint64_t limit_ns) {
  return __all_sync(0xffffffffu, mbar_wait_warp(bar, parity, abort_flag, status, code, limit_ns));
}

// ---- exchange of accumulators (cut along k) and results straight to memory -------------------------
// A piece of 32 columns by 128 rows, as the other pairs send it: 16 bytes of a row next to those of the next
// row, so that lanes (rows) write and read neighbouring addresses.
constexpr uint32_t kShareBytes = 128 * 32 * 4;
__device__ __forceinline__ void send8(uint32_t to, int row, int c8, const float (&f)[8]) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
    st_cluster_v4(to + ((2 * c8 + c) * 128 + row) * 16, __float_as_uint(f[4 * c]), __float_as_uint(f[4 * c + 1]),
                  __float_as_uint(f[4 * c + 2]), __float_as_uint(f[4 * c + 3]));
}
// The sum of all pairs' parts in their order; f holds this pair's.  Piece `local` of `each` a pair lies at
// from + (slot * each + local) pieces, slots being the other pairs in order.
__device__ __forceinline__ void join8(uint32_t from, int row, int c8, int splits, int share, int each, int local, float (&f)[8]) {
  float own[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    own[i] = f[i];
    f[i] = 0.0f;
  }
  for (int s = 0; s < splits; ++s) {
    if (s == share) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] += own[i];
    } else {
      const uint32_t at = from + uint32_t((s < share ? s : s - 1) * each + local) * kShareBytes + (2 * c8 * 128 + row) * 16;
      uint32_t w[8];
      ld_shared_v4(at, w[0], w[1], w[2], w[3]);
      ld_shared_v4(at + 128 * 16, w[4], w[5], w[6], w[7]);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] += __uint_as_float(w[i]);
    }
  }
}
// Eight columns of a row of a result, the first n of them in range.
template <typename T>
__device__ __forceinline__ void write8(char* base, int64_t rs, int64_t cs, int64_t row, int64_t col, int n, const float (&f)[8]) {
  T* to = reinterpret_cast<T*>(base) + row * rs + col * cs;
  if (n >= 8 && cs == 1 && (reinterpret_cast<uintptr_t>(to) & 15u) == 0) {
    if constexpr (sizeof(T) == 4) {
      reinterpret_cast<float4*>(to)[0] = make_float4(f[0], f[1], f[2], f[3]);
      reinterpret_cast<float4*>(to)[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
      *reinterpret_cast<uint4*>(to) = pack8<T>(f);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) to[i * cs] = from_f32<T>(f[i]);
  }
}
template <typename T>
__device__ __forceinline__ void read8(const char* base, int64_t rs, int64_t row, int64_t col, int n, float (&f)[8]) {
  const T* from = reinterpret_cast<const T*>(base) + row * rs + col;  // rows are 16-byte aligned, col a multiple of 8
  if (n >= 8) {
    unpack8<T>(*reinterpret_cast<const uint4*>(from), f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? to_f32(from[i]) : 0.0f;
  }
}

template <int kEpi, typename T>
__global__ void __launch_bounds__(kThreads, 1) cconv_pair_product_kernel(
    const __grid_constant__ PairMaps<kProductsOf<kEpi>> maps, const __grid_constant__ PairParams<kProductsOf<kEpi>> p) {
  extern __shared__ uint8_t smem_raw[];
  constexpr bool kEightBit = kEpi == kScaled;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t staging = base + p.stages * p.stage_bytes;
  const uint32_t scales = staging + kEpilogueWarps * p.pieces * kBoxBytes;
  const uint32_t bars = (scales + (kEightBit ? 2 * kEpilogueWarps * kScaleBytes : 0) + 7) & ~7u;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * p.stages;
  const uint32_t bar_tfull = bar_empty + 8 * p.stages, bar_tempty = bar_tfull + 16, bar_in = bar_tempty + 16;
  const uint32_t slot = bar_in + 8 * kEpilogueWarps;
  volatile int* abort_p = reinterpret_cast<volatile int*>(smem_raw + (slot + 4 - smem_u32(smem_raw)));

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t in_cluster = cluster_ctarank(), rank = in_cluster & 1, leader = in_cluster & ~1u;
  // uncut: the cluster is a pair, which goes through its tiles.  Cut: the cluster's pairs share one tile.
  const int share = int(in_cluster >> 1), cluster = int(blockIdx.x) / (2 * p.splits);
  const int stride = p.splits > 1 ? p.tiles : int(gridDim.x >> 1);

  if (threadIdx.x == 0) {
    *abort_p = 0;
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_tfull + 8 * i, 1);
      mbar_init(bar_tempty + 8 * i, 2 * kEpilogueWarps);
    }
    for (int i = 0; i < kEpilogueWarps; ++i) mbar_init(bar_in + 8 * i, 1);
    fence_barrier_init();
  }
  if (warp == 2) {
    pair_tmem_alloc(slot, kTmemCols);
    pair_tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // all CTAs' barriers are initialised
  tc_fence_after();
  uint32_t tmem;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));

  start_in_order();

  // 8-bit: the epilogue's sums take registers that the other warps do not need (128 x 80 + 256 x 208 of
  // the 384 x 168 that the block starts with)
  if (warp < 4) {
    if constexpr (kEightBit) asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 0 || warp == 3) {
      // One thread copies A, one B: a copy costs its thread some 150 clocks to issue, and a stage has two or three.
      const bool of_a = warp == 0;
      if (elect_one()) {
        uint32_t s = 0, ph = 0;
        const uint32_t full0 = cluster_map_shared(bar_full, leader);
        bool ok = true;
        for (int t = cluster; ok && t < p.tiles; t += stride) {
          const Tile tl = tile_of(p, t);
          const ProductParams& o = p.of[tl.of];
          const ProductMaps& om = maps.of[tl.of];
          const int row = of_a ? tl.m * 256 + int(rank) * 128
                               : p.paired ? tl.n * 128 : tl.n * o.block_n + int(rank) * (o.block_n >> 1);
          const int k0 = share * o.kb_part, k1 = min(o.kb_total, k0 + o.kb_part), kb_seg = o.kb_seg;
          const uint32_t bytes = of_a ? o.a_bytes : o.b_bytes;
          const bool kmajor = of_a ? o.a_kmajor : o.b_kmajor;
          const int boxes = kmajor ? 1 : int(bytes >> 13);
          const bool none = of_a && o.one_sided && rank;  // its rows are past the end
          const uint32_t expected = (o.one_sided ? 1 : 2) * o.a_bytes + 2 * o.b_bytes;
          const CUtensorMap* map0 = of_a ? &om.a[0] : &om.b[p.paired && rank];
          const CUtensorMap* map1 = of_a ? &om.a[1] : &om.b[1];
          uint32_t to = base + s * p.stage_bytes + (of_a ? 0 : p.a_stage);
          for (int kb = k0; kb < k1; ++kb) {
            if (!mbar_try_wait(bar_empty + 8 * s, ph ^ 1) &&
                !mbar_wait_slow(bar_empty + 8 * s, ph ^ 1, abort_p, p.status, kStatProducerWait, p.limit_ns)) {
              ok = false;
              break;
            }
            const bool seg = kb >= kb_seg;
            const int k = (seg ? kb - kb_seg : kb) * (kEightBit ? 128 : 64);
            const CUtensorMap* map = seg ? map1 : map0;
            const uint32_t bar = full0 + 8 * s;
            if (of_a && rank == 0) mbar_arrive_expect_tx(bar_full + 8 * s, expected);
            if (!none) {
              if (kmajor) {
                tma_load_2d_pair(to, map, k, row, bar);
              } else {
                for (int i = 0; i < boxes; ++i) tma_load_2d_pair(to + 8192 * i, map, row + 64 * i, k, bar);
              }
            }
            to += p.stage_bytes;
            if (++s == uint32_t(p.stages)) {
              s = 0;
              ph ^= 1;
              to -= p.stages * p.stage_bytes;
            }
          }
        }
      }
    } else if (warp == 1) {
      if (rank == 0) {
        const bool issue = elect_one();
        const uint16_t both = uint16_t(3u << leader);
        uint32_t s = 0, ph = 0, buf = 0, bph = 0;
        bool ok = true;
        for (int t = cluster; ok && t < p.tiles; t += stride) {
          const Tile tl = tile_of(p, t);
          const ProductParams& o = p.of[tl.of];
          const int k0 = share * o.kb_part, k1 = min(o.kb_total, k0 + o.kb_part);
          const uint64_t a_desc = o.a_desc, b_desc = o.b_desc;
          const uint32_t a_step = o.a_step, b_step = o.b_step, idesc = o.idesc;
          if constexpr (!kEightBit) {
            if (!wait_all(bar_tempty + 8 * buf, bph ^ 1, abort_p, p.status, kStatMmaWaitTmem, p.limit_ns)) break;
            tc_fence_after();
          }
          for (int kb = k0; kb < k1; ++kb) {
            if constexpr (kEightBit) {  // sums of one block of 128 a time
              if (!wait_all(bar_tempty + 8 * buf, bph ^ 1, abort_p, p.status, kStatMmaWaitTmem, p.limit_ns)) {
                ok = false;
                break;
              }
            }
            const uint32_t d = tmem + buf * 256;
            if (!wait_all(bar_full + 8 * s, ph, abort_p, p.status, kStatMmaWaitFull, p.limit_ns)) {
              ok = false;
              break;
            }
            tc_fence_after();
            // (a descriptor takes 18 bits of an address; above them lies the CTA's rank in its cluster)
            const uint32_t a = (base + s * p.stage_bytes) & 0x3ffffu;
            if (issue) {
              const uint64_t da = a_desc + (a >> 4), db = b_desc + ((a + p.a_stage) >> 4);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if constexpr (kEightBit) pair_mma_f8(d, da + j * 2, db + j * 2, idesc, j > 0);
                else pair_mma_f16(d, da + j * a_step, db + j * b_step, idesc, kb > k0 || j > 0);
              }
              pair_commit(bar_empty + 8 * s, both);
              if constexpr (kEightBit) pair_commit(bar_tfull + 8 * buf, both);
            }
            __syncwarp();
            if constexpr (kEightBit) {
              if (++buf == 2) buf = 0, bph ^= 1;
            }
            if (++s == uint32_t(p.stages)) s = 0, ph ^= 1;
          }
          if constexpr (!kEightBit) {
            if (issue && ok) pair_commit(bar_tfull + 8 * buf, both);
            __syncwarp();
            if (++buf == 2) buf = 0, bph ^= 1;
          }
        }
      }
    }
    if (p.splits > 1) {  // (see the epilogue)
      __syncwarp();
      cluster_sync_all();
      cluster_sync_all();
    }
  } else {
    if constexpr (kEightBit) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int q = warp & 3, half = (warp - 4) >> 2;
    const uint32_t mine = staging + (warp - 4) * p.pieces * kBoxBytes;
    const uint32_t in_bar = bar_in + 8 * (warp - 4);
    const uint32_t tempty0 = cluster_map_shared(bar_tempty, leader);
    const uint32_t lanes = tmem + (uint32_t(q * 32) << 16);
    uint32_t buf = 0, bph = 0, in_ph = 0, piece = 0;
    // The scales of 16 blocks of k from kb on, of tile t, on their way to half `b` of this warp's table.
    const uint32_t my_scales = scales + (warp - 4) * 2 * kScaleBytes;
    uint32_t sbuf = 0;
    auto fetch_scales = [&](const Tile& tl, int kb, uint32_t b) {
      const ProductParams& o = p.of[0];
      const int sub = lane >> 4, k = min(kb + (lane & 15), o.kb_total - 1);
      const int64_t r0 = int64_t(tl.m) * 256 + int(rank) * 128 + q * 32 + sub;
      const int rows = int(min(int64_t(32), o.M - r0));  // from r0 on; what lies past them reads as 0
      const float* from = p.row_scale + min(r0, o.M - 1) * p.row_rs + k * p.row_ks;
      uint32_t to = my_scales + b * kScaleBytes + (lane & 15) * 4 + sub * 68;
#pragma unroll
      for (int r = 0; r < 32; r += 2) {
        cp_async4(to + r * 68, from, r < rows);
        if (r + 2 < rows) from += 2 * p.row_rs;
      }
      const int64_t nb = min((int64_t(tl.n) * o.block_n + half * (o.block_n >> 1)) >> 7, (o.N - 1) >> 7);
      if (sub == 0) cp_async4(to + 32 * 68, p.col_scale + nb * p.col_rs + k * p.col_ks, true);
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    bool met = false;  // the cluster's two meetings are behind this warp
    Tile next = tile_of(p, cluster);
    if constexpr (kEightBit) fetch_scales(next, share * p.of[0].kb_part, 0);
    for (int t = cluster; t < p.tiles; t += stride) {
      const Tile tl = next;
      next = tile_of(p, min(t + stride, p.tiles - 1));
      const ProductParams& o = p.of[tl.of];
      const CUtensorMap* out_map = &maps.of[tl.of].out;
      const int row0 = tl.m * 256 + int(rank) * 128 + q * 32;
      uint32_t acc = lanes + buf * 256;
      auto wait_sums = [&]() {
        if (!wait_all(bar_tfull + 8 * buf, bph, abort_p, p.status, kStatEpilogueWait, p.limit_ns)) return false;
        tc_fence_after();
        return true;
      };
      auto release_sums = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tempty0 + 8 * buf);
      };
      if constexpr (!kEightBit) {
        if (p.splits > 1) {  // cut: results straight to memory
          // Columns go in pieces of 32; the pair `owner` finishes `each` neighbouring ones (of both
          // g and u when paired).  The two halves of the warps take turns.
          if (!wait_sums()) break;
          const int all = p.paired ? 4 : o.block_n >> 5, each = all / p.splits, sent = p.paired ? 2 * each : each;
          const int row = q * 32 + lane;
          cluster_sync_all();  // every pair's operands are used up: their place takes the pieces
          for (int i = half; i < all; i += 2) {
            const int owner = i / each;
            if (owner == share) continue;
            const uint32_t to = cluster_map_shared(base, uint32_t(2 * owner) + rank) +
                                uint32_t((share < owner ? share : share - 1) * sent + i - owner * each) * kShareBytes;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              float f[8];
              load_sums8(acc + i * 32 + c * 8, f);
              send8(to, row, c, f);
              if (p.paired) {
                load_sums8(acc + 128 + i * 32 + c * 8, f);
                send8(to + each * kShareBytes, row, c, f);
              }
            }
          }
          cluster_sync_all();  // all pieces have come
          met = true;
          for (int i = share * each + half; i < (share + 1) * each; i += 2) {
            const int local = i - share * each;
            const int64_t r = row0 + lane, col = int64_t(tl.n) * (p.paired ? 128 : o.block_n) + i * 32;
            const int cols = r < o.M ? int(min(int64_t(32), o.N - col)) : 0;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              const int64_t at = col + c * 8;
              const int n = cols - c * 8;
              float f[8];
              load_sums8(acc + i * 32 + c * 8, f);
              join8(base, row, c, p.splits, share, sent, local, f);
              if constexpr (kEpi == kStore) {
                write8<T>(p.out[0], p.out_rs[0], p.out_cs[0], r, at, n, f);
              } else if constexpr (kEpi == kGated) {
                float u[8];
                load_sums8(acc + 128 + i * 32 + c * 8, u);
                join8(base, row, c, p.splits, share, sent, each + local, u);
                if (p.save) {
                  write8<T>(p.out[1], p.out_rs[1], p.out_cs[1], r, at, n, f);
                  write8<T>(p.out[2], p.out_rs[2], p.out_cs[2], r, at, n, u);
                }
                gate(p.act, f, u);
                write8<T>(p.out[0], p.out_rs[0], p.out_cs[0], r, at, n, f);
              } else {
                float g[8], u[8];
                read8<T>(p.in[0], p.in_rs[0], r, at, n, g);
                read8<T>(p.in[1], p.in_rs[1], r, at, n, u);
                gate_backward(p.act, f, g, u);
                write8<T>(p.out[0], p.out_rs[0], p.out_cs[0], r, at, n, g);
                write8<T>(p.out[1], p.out_rs[1], p.out_cs[1], r, at, n, f);
                write8<T>(p.out[2], p.out_rs[2], p.out_cs[2], r, at, n, u);
              }
            }
          }
          break;  // there is one tile
        }
      }
      if constexpr (kEpi == kStore) {
        if (!wait_sums()) break;
        const int cols = o.block_n >> 1;
        for (int c = 0; c < cols; c += 64) {
          const bool narrow = cols < 64;  // 64 columns a tile: one half of the warps takes them all
          if (narrow && half) {
            release_sums();
            break;
          }
          const int at = narrow ? 0 : half * cols + c;
          float f[32], g[32];
          load_sums(acc + at, f);
          load_sums(acc + at + 32, g);
          if (c + 64 >= cols) release_sums();
          const uint32_t to = mine + piece * kBoxBytes;
          if (lane == 0) bulk_wait_group_read<1>();
          __syncwarp();
          stage32<T>(to, lane, 0, f);
          stage32<T>(to, lane, 4, g);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            const int col = tl.n * o.block_n + at;
            if (row0 < o.M && col < o.N) tma_store_2d(out_map, to, col, row0);
            bulk_commit_group();
          }
          piece ^= 1;
        }
      } else if constexpr (kEpi == kGated) {
        if (!wait_sums()) break;
        const int col = tl.n * 128 + half * 64;
        if (lane == 0) bulk_wait_group_read<0>();
        __syncwarp();
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          float g[32], u[32];
          load_sums(acc + half * 64 + c * 32, g);
          load_sums(acc + 128 + half * 64 + c * 32, u);
          if (c == 1) release_sums();
          if (p.save) {
            stage32<T>(mine + kBoxBytes, lane, c * 4, g);
            stage32<T>(mine + 2 * kBoxBytes, lane, c * 4, u);
          }
          gate(p.act, g, u);
          stage32<T>(mine, lane, c * 4, g);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (row0 < o.M && col < o.N) {
            tma_store_2d(out_map, mine, col, row0);
            if (p.save) {
              tma_store_2d(&maps.out1, mine + kBoxBytes, col, row0);
              tma_store_2d(&maps.out2, mine + 2 * kBoxBytes, col, row0);
            }
          }
          bulk_commit_group();
        }
      } else if constexpr (kEpi == kGatedBackward) {
        const int cols = o.block_n >> 1;
        bool first = true, ok = true;
        for (int c = 0; c < cols; c += 64) {
          const int col = tl.n * o.block_n + half * cols + c;
          if (lane == 0) {
            bulk_wait_group_read<0>();
            mbar_arrive_expect_tx(in_bar, 2 * kBoxBytes);
            tma_load_2d(mine, &maps.in[0], col, row0, in_bar);
            tma_load_2d(mine + kBoxBytes, &maps.in[1], col, row0, in_bar);
          }
          if (first && !(ok = wait_sums())) break;
          first = false;
          if (!(ok = wait_all(in_bar, in_ph, abort_p, p.status, kStatEpilogueWait, p.limit_ns))) break;
          in_ph ^= 1;
#pragma unroll 1
          for (int j = 0; j < 2; ++j) {
            float d[32], g[32], u[32];
            load_sums(acc + half * cols + c + j * 32, d);
            if (j == 1 && c + 64 >= cols) release_sums();
            unstage32<T>(mine, lane, j * 4, g);
            unstage32<T>(mine + kBoxBytes, lane, j * 4, u);
            gate_backward(p.act, d, g, u);
            stage32<T>(mine, lane, j * 4, g);
            stage32<T>(mine + kBoxBytes, lane, j * 4, d);
            stage32<T>(mine + 2 * kBoxBytes, lane, j * 4, u);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (row0 < o.M && col < o.N) {
              tma_store_2d(out_map, mine, col, row0);
              tma_store_2d(&maps.out1, mine + kBoxBytes, col, row0);
              tma_store_2d(&maps.out2, mine + 2 * kBoxBytes, col, row0);
            }
            bulk_commit_group();
          }
        }
        if (!ok) break;
      } else {
        // Each block's sums are scaled and added up in registers (a row of half the columns a thread),
        // beside the MMAs of the next block: 128 columns are 64 two-wide multiply-adds.
        const int cols = o.block_n >> 1;
        const int k0 = share * o.kb_part, k1 = min(o.kb_total, k0 + o.kb_part);
        uint64_t sum[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) sum[i] = 0;
        auto scale_of = [&](int kb) {
          if (((kb - k0) & 15) == 0) {
            // this half of the table has come; the other is free, as every lane is past its last use
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
            const bool on = kb + 16 < k1;
            fetch_scales(on ? tl : next, on ? kb + 16 : k0, sbuf ^ 1);
            sbuf ^= 1;
          }
          const uint32_t at = my_scales + (sbuf ^ 1) * kScaleBytes + ((kb - k0) & 15) * 4;
          return ld_shared_f32(at + lane * 68) * ld_shared_f32(at + 32 * 68);
        };
        bool ok = true;
        for (int kb = k0; kb < k1; ++kb) {
          const float f0 = scale_of(kb);
          const uint64_t scale = pair_of(f0, f0);
          if (!(ok = wait_sums())) break;
          // 64 columns at a time; the second 64 are on their way while the first are added up
          uint32_t f[2][32];
          auto add = [&](int c) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              sum[c * 16 + i] = fma2(pair_of(__uint_as_float(f[c & 1][2 * i]), __uint_as_float(f[c & 1][2 * i + 1])), scale,
                                     sum[c * 16 + i]);
          };
          tmem_ld_32x32b_x32(acc + half * cols, f[0]);
          tmem_ld_32x32b_x32(acc + half * cols + 32, f[1]);
          tmem_ld_wait(f[0]);
          tmem_ld_hold(f[1]);
          if (cols == 64) release_sums();
          add(0);
          if (cols > 64) tmem_ld_32x32b_x32(acc + half * cols + 64, f[0]);
          add(1);
          if (cols > 64) {
            tmem_ld_32x32b_x32(acc + half * cols + 96, f[1]);
            tmem_ld_wait(f[0]);
            tmem_ld_hold(f[1]);
            release_sums();
            add(2);
            add(3);
          }
          if (++buf == 2) buf = 0, bph ^= 1;
          acc = lanes + buf * 256;
        }
        if (!ok) break;
        auto piece32 = [&](int c, float (&f)[32]) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 v = halves_of(sum[c * 16 + i]);
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
          }
        };
        auto piece8 = [&](int c, float (&f)[8]) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 v = halves_of(sum[c * 4 + i]);
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
          }
        };
        if (p.splits > 1) {  // as above, with the sums in registers
          const int each = (o.block_n >> 5) / p.splits, row = q * 32 + lane, first = half * (cols >> 5);
          cluster_sync_all();
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int i = first + c, owner = i / each;
            if (c * 32 < cols && owner != share) {
              const uint32_t to = cluster_map_shared(base, uint32_t(2 * owner) + rank) +
                                  uint32_t((share < owner ? share : share - 1) * each + i - owner * each) * kShareBytes;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float f[8];
                piece8(c * 4 + e, f);
                send8(to, row, e, f);
              }
            }
          }
          cluster_sync_all();
          met = true;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int i = first + c;
            if (c * 32 < cols && i / each == share) {
              const int64_t r = row0 + lane, col = int64_t(tl.n) * o.block_n + i * 32;
              const int n = r < o.M ? int(min(int64_t(32), o.N - col)) : 0;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float f[8];
                piece8(c * 4 + e, f);
                join8(base, row, e, p.splits, share, each, i - share * each, f);
                write8<T>(p.out[0], p.out_rs[0], p.out_cs[0], r, col + e * 8, n - e * 8, f);
              }
            }
          }
          break;
        }
        constexpr int kWidth = 128 / int(sizeof(T));  // columns of a piece
#pragma unroll
        for (int c = 0; c < 128; c += kWidth) {
          if (c < cols) {
            if (lane == 0) bulk_wait_group_read<0>();
            __syncwarp();
            float f[32];
            piece32(c / 32, f);
            if constexpr (sizeof(T) == 4) {
              stage_f32(mine, lane, f);
            } else {
              stage32<T>(mine, lane, 0, f);
              piece32(c / 32 + 1, f);
              stage32<T>(mine, lane, 4, f);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              const int col = tl.n * o.block_n + half * cols + c;
              if (row0 < o.M && col < o.N) tma_store_2d(out_map, mine, col, row0);
              bulk_commit_group();
            }
          }
        }
        continue;  // the buffers were handed on block by block
      }
      if (++buf == 2) buf = 0, bph ^= 1;
    }
    if (p.splits > 1 && !met) {  // gave up on the way: the others are not kept waiting
      __syncwarp();
      cluster_sync_all();
      cluster_sync_all();
    }
    if constexpr (kEightBit) asm volatile("cp.async.wait_all;" ::: "memory");
    if (lane == 0) bulk_wait_group<0>();
  }

  // A wait that ran out raised the flag a whole limit after the last copy or MMA was issued; the other
  // roles leave within a poll of it.  A short pause lets what they issued last come to its end.
  __syncwarp();
  __syncthreads();
  if (*abort_p) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000) {
    }
  }
  __syncwarp();
  tc_fence_before();
  cluster_sync_all();  // nothing arrives at, or reads, another CTA's shared memory any more
  tc_fence_after();
  if (warp == 2) pair_tmem_dealloc(tmem, kTmemCols);
}

template <int kEpi, typename T>
cudaError_t launch_pair(const PairMaps<kProductsOf<kEpi>>& maps, const PairParams<kProductsOf<kEpi>>& p, int sms,
                        cudaStream_t s) {
  auto f = cconv_pair_product_kernel<kEpi, T>;
  static bool ready[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!__atomic_load_n(&ready[dev & 63], __ATOMIC_ACQUIRE)) {
    e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmemMost));
    if (e != cudaSuccess) return e;
    __atomic_store_n(&ready[dev & 63], true, __ATOMIC_RELEASE);
  }
  const int pairs = p.splits > 1 ? p.tiles * p.splits : p.tiles < sms / 2 ? p.tiles : sms / 2;
  // All of an SM's shared memory, needed or not: no other block may share the SM, as it could hold the tensor
  // memory that one CTA of a cluster waits for while that block's kernel waits for another CTA of the cluster.
  const size_t smem = kSmemMost;
  return launch(f, dim3(unsigned(2 * pairs)), kThreads, smem, 2 * p.splits, s, maps, p);
}

int encode_operand(CUtensorMap* tm, const Operand& o, int es, int dtype, int rows_box) {
  if (es == 1) return encode_map(tm, o.p, 1, dtype, o.k, o.rows, o.pitch, 128, rows_box);
  return o.kmajor ? encode_map(tm, o.p, 2, dtype, o.k, o.rows, o.pitch, 64, rows_box)
                  : encode_map(tm, o.p, 2, dtype, o.rows, o.k, o.pitch, 64, 64);
}

template <int kEpi>
int run_as(const Launch& l, int sms, cudaStream_t s) {
  constexpr int kProducts = kProductsOf<kEpi>;
  constexpr bool kEight = kEpi == kScaled;
  PairMaps<kProducts> maps;
  PairParams<kProducts> q;
  int rc = block_status_word(&q.status);
  if (rc != CCONV_OK) return rc;
  const int es = type_bytes(l.dtype);
  uint32_t a_most = 0, b_most = 0;
  q.tiles = 0;
  q.count = l.count;
  q.splits = l.splits;
  for (int i = 0; i < l.count; ++i) {
    const Product& p = l.of[i];
    ProductParams& o = q.of[i];
    ProductMaps& m = maps.of[i];
    o.tiles_m = int(cdiv64(p.M, 256));
    o.tiles_n = int(cdiv64(p.N, p.paired ? 128 : p.block_n));
    o.first = q.tiles;
    q.tiles += o.tiles_m * o.tiles_n;
    o.kb_seg = int(cdiv64(p.K, kEight ? 128 : 64));
    o.kb_total = o.kb_seg * (p.segments ? 2 : 1);
    o.kb_part = int(cdiv64(o.kb_total, l.splits));
    o.block_n = p.block_n;
    o.b_bytes = uint32_t(p.block_n / 2) * 128;
    o.a_bytes = uint32_t(a_rows_of(p)) * 128;
    o.one_sided = p.M <= 128;
    a_most = std::max(a_most, o.a_bytes);
    b_most = std::max(b_most, o.b_bytes);
    o.a_kmajor = p.a[0].kmajor;
    o.b_kmajor = p.b[0].kmajor;
    o.a_desc = swizzled_desc(p.a[0].kmajor, 8192);
    o.b_desc = swizzled_desc(p.b[0].kmajor, 8192);
    o.a_step = p.a[0].kmajor ? 32 >> 4 : 2048 >> 4;
    o.b_step = p.b[0].kmajor ? 32 >> 4 : 2048 >> 4;
    const uint32_t type = !kEight && l.dtype == CCONV_TYPE_BF16 ? 1u : 0u;  // (8 bits: 0 is e4m3)
    // instruction descriptor: D fp32, types of A and B, their orders (1: rows contiguous), N / 8, M / 16
    o.idesc = (1u << 4) | (type << 7) | (type << 10) | (uint32_t(!p.a[0].kmajor) << 15) |
              (uint32_t(!p.b[0].kmajor) << 16) | (uint32_t(p.block_n >> 3) << 17) | (uint32_t(256 >> 4) << 24);
    o.M = p.M;
    o.N = p.N;
    for (int j = 0; j < 2 && rc == CCONV_OK; ++j) {
      if (j == 0 || p.segments) rc = encode_operand(&m.a[j], p.a[j], kEight ? 1 : 2, l.dtype, a_rows_of(p));
      if (rc == CCONV_OK && (j == 0 || p.segments || p.paired)) rc = encode_operand(&m.b[j], p.b[j], kEight ? 1 : 2, l.dtype, p.block_n / 2);
    }
    if (rc == CCONV_OK && !l.cut()) rc = encode_map(&m.out, p.out[0].p, es, l.dtype, p.N, p.M, p.out[0].rs, 128 / es, 32);
    if (rc != CCONV_OK) return rc;
  }
  const Product& p = l.of[0];
  for (int i = 0; i < 3; ++i) {
    q.out[i] = static_cast<char*>(const_cast<void*>(p.out[i].p));
    q.out_rs[i] = p.out[i].rs;
    q.out_cs[i] = p.out[i].cs;
  }
  for (int i = 0; i < 2; ++i) {
    q.in[i] = static_cast<const char*>(p.in[i].p);
    q.in_rs[i] = p.in[i].rs;
  }
  if constexpr (kEpi == kGated || kEpi == kGatedBackward) {
    CUtensorMap* more_maps[4] = {&maps.out1, &maps.out2, &maps.in[0], &maps.in[1]};
    const Mat* mats[4] = {&p.out[1], &p.out[2], &p.in[0], &p.in[1]};
    for (int i = 0; i < 4 && !l.cut(); ++i)
      if (mats[i]->p && (rc = encode_map(more_maps[i], mats[i]->p, es, l.dtype, p.N, p.M, mats[i]->rs, 64, 32))) return rc;
  }
  q.a_stage = a_most;
  q.stage_bytes = a_most + b_most;
  q.pieces = uint32_t(pieces_of(l));
  q.stages = stages_of(l, a_most, b_most);
  q.paired = p.paired;
  q.act = l.act;
  q.save = l.save;
  q.row_scale = static_cast<const float*>(l.row_scale.p);
  q.row_rs = l.row_scale.rs;
  q.row_ks = l.row_scale.cs;
  q.col_scale = static_cast<const float*>(l.col_scale.p);
  q.col_rs = l.col_scale.rs;
  q.col_ks = l.col_scale.cs;
  q.limit_ns = block_wait_limit_ns();
  cudaError_t e;
  if (l.dtype == CCONV_TYPE_BF16) e = launch_pair<kEpi, __nv_bfloat16>(maps, q, sms, s);
  else if (l.dtype == CCONV_TYPE_FP16) e = launch_pair<kEpi, __half>(maps, q, sms, s);
  else if constexpr (kEight) e = launch_pair<kEpi, float>(maps, q, sms, s);
  else return CCONV_EUNSUPPORTED;
  return block_cuda_error(e, "cconv_pair_product_kernel");
}

// Clocks of a k block of a tile, and of what begins and ends a launch or, where cut, a round of tiles, as
// measured on products of 64 to 2048 rows (back to back, operands in L2): a block costs the tensor cores'
// 2 clocks a column, or 340 (390 with rows of B contiguous) that a stage takes to come and go; 8-bit sums are
// scaled at 3.5 clocks a column with 220 a block.  8 us a launch, 11 and 12.5 a round of 2 and 4 pairs a tile.
double block_clocks(const Launch& l, const Product& p) {
  if (l.epilogue == kScaled) return 220.0 + 2.65 * p.block_n;
  return std::max(2.0 * p.block_n, p.b[0].kmajor ? 340.0 : 390.0);
}
double fixed_clocks(const Launch& l, int block_n) {
  const double epilogue = l.epilogue == kGatedBackward ? (block_n == 256 ? 11000.0 : 5000.0)
                          : l.epilogue == kScaled && l.splits > 1 ? 8000.0 : 0.0;
  return (l.splits == 1 ? 14600.0 : l.splits == 2 ? 20000.0 : 23000.0) + epilogue;
}

// Copies of rows that are contiguous on both sides, several at once: blockIdx.z is the copy, 64 threads by 4
// rows a block, 4 pieces of 16 bytes a thread.  Rows that begin anywhere are written in the target's pieces,
// each from the five words of the source that it lies in; pieces that a row's ends cut, and those whose words would
// reach out of the source, go byte by byte (two operands of 4000 x 4095 and 4095 x 4095 bytes: 35 us; with the
// widest accesses that both sides' alignment allows, which is a byte there, 70 us).
struct RowCopy {
  const char* from;
  char* to;
  int64_t from_pitch, to_pitch, rows, bytes;  // pitches and row length in bytes
  int aligned;                                // all of them, and the addresses, to 16 bytes
};
struct RowCopies {
  RowCopy of[kMostCopies];
};
__device__ __forceinline__ void copy_aligned_row(const RowCopy& c, int64_t r, int64_t x0) {
  const uint4* src = reinterpret_cast<const uint4*>(c.from + r * c.from_pitch);
  uint4* dst = reinterpret_cast<uint4*>(c.to + r * c.to_pitch);
  uint4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (x0 + 64 * i < c.bytes / 16) v[i] = src[x0 + 64 * i];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (x0 + 64 * i < c.bytes / 16) dst[x0 + 64 * i] = v[i];
}
__device__ __forceinline__ void copy_row(const RowCopy& c, int64_t r, int64_t x0) {
  const char* src = c.from + r * c.from_pitch;
  char* dst = c.to + r * c.to_pitch;
  const uintptr_t first = reinterpret_cast<uintptr_t>(c.from),
                  last = first + uintptr_t((c.rows - 1) * c.from_pitch + c.bytes);  // the source, all of it
  const int64_t lead = int64_t(reinterpret_cast<uintptr_t>(dst) & 15);
  uint32_t w[4][5];
  bool whole[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = (x0 + 64 * i) * 16 - lead;  // of the piece, from the row's start
    const uintptr_t a = reinterpret_cast<uintptr_t>(src + at), words = a & ~uintptr_t(3);
    whole[i] = at >= 0 && at + 16 <= c.bytes && words >= first && words + 20 <= last;
    if (whole[i]) {
#pragma unroll
      for (int k = 0; k < 5; ++k) w[i][k] = reinterpret_cast<const uint32_t*>(words)[k];
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = (x0 + 64 * i) * 16 - lead;
    if (whole[i]) {
      const uint32_t by = uint32_t(reinterpret_cast<uintptr_t>(src + at) & 3) * 8;
      *reinterpret_cast<uint4*>(dst + at) =
          make_uint4(__funnelshift_r(w[i][0], w[i][1], by), __funnelshift_r(w[i][1], w[i][2], by),
                     __funnelshift_r(w[i][2], w[i][3], by), __funnelshift_r(w[i][3], w[i][4], by));
    } else {
      for (int64_t k = max(at, int64_t(0)); k < min(at + 16, c.bytes); ++k) dst[k] = src[k];
    }
  }
}
__global__ void __launch_bounds__(256) cconv_copy_rows_kernel(const __grid_constant__ RowCopies copies) {
  start_in_order();
  const RowCopy& c = copies.of[blockIdx.z];
  const int64_t pieces = (c.bytes + (c.aligned ? 15 : 30)) / 16;  // unaligned: at most
  for (int64_t x0 = int64_t(blockIdx.x) * 256 + (threadIdx.x & 63); x0 < pieces; x0 += int64_t(gridDim.x) * 256) {
    for (int64_t r = int64_t(blockIdx.y) * 4 + (threadIdx.x >> 6); r < c.rows; r += int64_t(gridDim.y) * 4) {
      if (c.aligned) copy_aligned_row(c, r, x0);
      else copy_row(c, r, x0);
    }
  }
}

// 32 x 32 elements a block through shared memory: read along the source's short stride, written along
// the target's.
template <typename E>
__global__ void __launch_bounds__(256) cconv_copy_kernel(Mat from, Mat to, int64_t rows, int64_t cols) {
  __shared__ E tile[32][33];
  start_in_order();
  const E* src = static_cast<const E*>(from.p);
  E* dst = static_cast<E*>(const_cast<void*>(to.p));
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int64_t c0 = int64_t(blockIdx.x) * 32;
  for (int64_t r0 = int64_t(blockIdx.y) * 32; r0 < rows; r0 += int64_t(gridDim.y) * 32) {
    const bool by_rows = from.rs < from.cs;  // neighbours in memory are rows
    for (int i = y; i < 32; i += 8) {
      const int r = by_rows ? x : i, c = by_rows ? i : x;
      if (r0 + r < rows && c0 + c < cols) tile[r][c] = src[(r0 + r) * from.rs + (c0 + c) * from.cs];
    }
    __syncthreads();
    const bool to_rows = to.rs < to.cs;
    for (int i = y; i < 32; i += 8) {
      const int r = to_rows ? x : i, c = to_rows ? i : x;
      if (r0 + r < rows && c0 + c < cols) dst[(r0 + r) * to.rs + (c0 + c) * to.cs] = tile[r][c];
    }
    __syncthreads();
  }
}

}  // namespace

uint64_t block_wait_limit_ns() {
  const char* v = std::getenv("CCONV_WAIT_LIMIT_MS");
  return uint64_t(v && *v ? std::atoi(v) : 1000) * 1000000ull;
}

int block_status_word(int** word) {
  static int* words[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return block_cuda_error(e, "cudaGetDevice");
  *word = __atomic_load_n(&words[dev & 63], __ATOMIC_ACQUIRE);
  if (*word) return CCONV_OK;
  void* p = nullptr;
  e = cudaGetSymbolAddress(&p, g_block_status);
  *word = static_cast<int*>(p);
  if (e == cudaSuccess) __atomic_store_n(&words[dev & 63], *word, __ATOMIC_RELEASE);
  return block_cuda_error(e, "cudaGetSymbolAddress");
}

namespace {
// Clusters of 2 * splits CTAs that run at one time: GPCs whose SMs a cluster does not divide leave some over
// (a B200 with 148 SMs: 74 of 2, 33 of 4, 15 of 8).
int cluster_slots(int splits, int sms) {
  static int known[64][3] = {};
  int dev = 0;
  const int which = splits == 1 ? 0 : splits == 2 ? 1 : 2, guess = std::max(1, sms / (2 * splits) - (splits > 1 ? 1 << which : 0));
  if (cudaGetDevice(&dev) != cudaSuccess) return guess;
  int n = __atomic_load_n(&known[dev & 63][which], __ATOMIC_RELAXED);
  if (n == 0) {
    auto f = cconv_pair_product_kernel<kStore, __nv_bfloat16>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(2 * splits * sms));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemMost;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(2 * splits);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmemMost)) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, f, &cfg) != cudaSuccess || n <= 0) {
      cudaGetLastError();
      n = guess;
    }
    __atomic_store_n(&known[dev & 63][which], n, __ATOMIC_RELAXED);
  }
  return n;
}
}  // namespace

double launch_clocks(const Launch& l, int sms) {
  const int es = l.epilogue == kScaled ? 1 : 2;
  const int slots = cluster_slots(l.splits, sms);
  double all = 0, longest = 0, bytes = 0;
  int64_t tiles = 0;
  for (int i = 0; i < l.count; ++i) {
    const Product& p = l.of[i];
    const int64_t n = cdiv64(p.M, 256) * cdiv64(p.N, p.paired ? 128 : p.block_n);
    const double c = double(cdiv64(cdiv64(p.K, 128 / es) * (p.segments ? 2 : 1), l.splits)) * block_clocks(l, p) + 600.0;
    tiles += n;
    all += double(n) * c;
    longest = std::max(longest, c);
    bytes += double(es) * (double(p.M + p.N * (p.paired ? 2 : 1)) * double(p.K) * (p.segments ? 2 : 1) + double(p.M) * double(p.N));
  }
  const double least = bytes / 3500.0;  // HBM, per clock
  const double fixed = fixed_clocks(l, l.of[0].block_n), rounds = double(cdiv64(tiles, slots));
  if (l.splits > 1) return std::max(least, rounds * (longest + fixed));
  if (l.count == 1) return std::max(least, rounds * longest) + fixed;
  return std::max(least, all / slots + 0.9 * longest) + fixed;
}

namespace {
void cut(Launch* l, int block_n, int splits) {
  Product& p = l->of[0];
  p.block_n = block_n;
  l->splits = splits;
}
}  // namespace

void choose_cut(Launch* l, int sms, bool few_columns) {
  Product& p = l->of[0];
  const int es = l->epilogue == kScaled ? 1 : 2;
  const int64_t kb = cdiv64(p.K, 128 / es) * (p.segments ? 2 : 1);
  int force_n = 0, force_s = 0;  // diagnostics: columns of a tile, pairs that share it
  if (const char* v = std::getenv("CCONV_BLOCK_CUT"))
    if (std::sscanf(v, "%d,%d", &force_n, &force_s) != 2) force_n = force_s = 0;
  double best = 0;
  int best_n = 0, best_s = 1;
  for (int n = 256; n >= 64; n /= 2) {
    if (p.paired && n != 256) continue;
    if (n == 64 && (!few_columns || !p.b[0].kmajor)) continue;
    for (int s = 1; s <= 4; s *= 2) {
      if (s > 1 && (s - 1) * cdiv64(kb, s) >= kb) continue;      // every pair has a part
      if ((p.paired ? 128 : n) / 32 < s) continue;                // and 32 columns to finish
      cut(l, n, s);
      double c = launch_clocks(*l, sms);
      if (n == force_n) c *= 1e-3;
      if (s == force_s) c *= 1e-3;
      if (best_n == 0 || c < best) best = c, best_n = n, best_s = s;
    }
  }
  cut(l, best_n, best_s);
}

int run_products(const Launch& l, int sms, cudaStream_t s) {
  if (l.epilogue == kStore) return run_as<kStore>(l, sms, s);
  if (l.epilogue == kGated) return run_as<kGated>(l, sms, s);
  if (l.epilogue == kGatedBackward) return run_as<kGatedBackward>(l, sms, s);
  return run_as<kScaled>(l, sms, s);
}

bool copies_rows(const Mat& from, const Mat& to) { return from.cs == 1 && to.cs == 1; }

cudaError_t run_row_copies(const Copy* copies, int n, cudaStream_t s) {
  RowCopies c{};
  int64_t x = 1, y = 1;
  for (int i = 0; i < n; ++i) {
    const Copy& k = copies[i];
    RowCopy& r = c.of[i];
    r.from = static_cast<const char*>(k.from.p);
    r.to = static_cast<char*>(const_cast<void*>(k.to.p));
    r.rows = k.rows;
    r.bytes = k.cols * k.es;
    r.from_pitch = k.from.rs * k.es;
    r.to_pitch = k.to.rs * k.es;
    uintptr_t all = reinterpret_cast<uintptr_t>(r.from) | reinterpret_cast<uintptr_t>(r.to) | uintptr_t(r.bytes);
    if (r.rows > 1) all |= uintptr_t(r.from_pitch) | uintptr_t(r.to_pitch);
    r.aligned = (all & 15) == 0;
    x = std::max(x, cdiv64((r.bytes + 30) / 16, 256));
    y = std::max(y, cdiv64(r.rows, 4));
  }
  const dim3 grid(unsigned(std::min<int64_t>(x, 65535)), unsigned(std::min<int64_t>(y, 16384)), unsigned(n));
  return launch(cconv_copy_rows_kernel, grid, 256, 0, 1, s, c);
}

cudaError_t run_copy(const Copy& k, cudaStream_t s) {
  const int64_t y = cdiv64(k.rows, 32);
  const dim3 grid(unsigned(cdiv64(k.cols, 32)), unsigned(y < 65535 ? y : 65535));
  if (k.es == 1) return launch(cconv_copy_kernel<uint8_t>, grid, 256, 0, 1, s, k.from, k.to, k.rows, k.cols);
  if (k.es == 4) return launch(cconv_copy_kernel<uint32_t>, grid, 256, 0, 1, s, k.from, k.to, k.rows, k.cols);
  return launch(cconv_copy_kernel<uint16_t>, grid, 256, 0, 1, s, k.from, k.to, k.rows, k.cols);
}

}  // namespace cconv
