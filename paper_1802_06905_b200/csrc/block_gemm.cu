// Products of the feed-forward block on pairs of CTAs.
//
// C = A B^T over a 256 x block_n tile a pair: each CTA keeps 128 rows of A and half the rows of B in shared
// memory (64 elements of k a stage), one thread of the first CTA issues the MMAs of both (M = 256), and
// each CTA's accumulators (128 x block_n, fp32) lie in its own tensor memory, twice, so that a tile's
// epilogue runs beside the next tile's main loop.  A pair reads (256 + block_n) rows of k from L2 for
// 256 x block_n products, half of what two CTAs on tiles of their own would: at 128 x 256 a CTA draws 96
// bytes a clock, a pair of CTAs at 256 x 256 64 bytes a clock each, below what L2 delivers to an SM.
//
// Roles: warp 0 copies (TMA), warp 1 of the first CTA issues MMAs, warp 2 owns the tensor memory, warps
// 4-11 are the epilogue (two for each quarter of the lanes, half of the columns each).
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

__device__ int g_block_status;

struct PairParams {
  int tiles_m, tiles_n, tiles_m0;  // tiles_m0: rows of tiles of the first stacked product
  int splits, kb_total, kb_split, kb_seg;
  int block_n, stages;
  uint32_t b_bytes;                // a stage of B in one CTA
  uint32_t a_kmajor, b_kmajor, paired;
  uint64_t a_desc, b_desc;
  uint32_t a_step, b_step;         // descriptor step of 16 elements of k (16-byte units)
  uint32_t idesc;
  int64_t M, N;
  int act, save, more;
  float* partial;
  int64_t pitch, slice;
  // 8-bit operands: scale of row r (or of 128 rows) and k block kb at row_scale[i * row_rs + kb * row_ks]
  const float *row_scale, *col_scale;
  int64_t row_rs, row_ks, col_rs, col_ks;
  int* status;
  uint64_t limit_ns;
};
struct PairMaps {
  CUtensorMap a[2], b[2], out[3], in[2];
};

// Tile t of the launch: share of k, row and column of tiles.  Tiles run down groups of 8 rows of tiles,
// so that the pairs at work at one time read few different rows of A and B.
struct Tile {
  int split, m, n;
};
__device__ __forceinline__ Tile tile_of(const PairParams& p, int t) {
  Tile r;
  r.split = t % p.splits;
  t /= p.splits;
  const int group = 8 * p.tiles_n;
  const int first = t / group * 8;
  const int rows = min(8, p.tiles_m - first);
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
__device__ __forceinline__ void unstage32(uint32_t base, int r, int c0, float (&f)[32]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint32_t w[4];
    ld_shared_v4(chunk_at(base, r, c0 + c), w[0], w[1], w[2], w[3]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = unpack2<T>(w[i]);
      f[8 * c + 2 * i] = v.x;
      f[8 * c + 2 * i + 1] = v.y;
    }
  }
}

// Pieces that an epilogue warp stages.
template <int kEpi>
constexpr int kPieces = kEpi == kStore ? 2 : kEpi == kScaled ? 1 : kEpi == kPartial || kEpi == kScaledPartial ? 0 : 3;
int staged_pieces(int epi) {
  return epi == kStore ? 2 : epi == kScaled ? 1 : epi == kPartial || epi == kScaledPartial ? 0 : 3;
}
// Scales of 8-bit rows that an epilogue warp keeps: 16 blocks of k of its 32 rows and of its columns
// (row 32), the 16 in use and the next 16; a pitch of 17 words keeps the lanes on different banks.
constexpr uint32_t kScaleBytes = 33 * 17 * 4;
uint32_t scale_bytes(int epi) { return epi == kScaled ? 2 * kEpilogueWarps * kScaleBytes : 0; }
template <int kEpi>
constexpr bool kEightBit = kEpi == kScaled || kEpi == kScaledPartial;

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

template <int kEpi, typename T>
__global__ void __launch_bounds__(kThreads, 1) cconv_pair_product_kernel(const __grid_constant__ PairMaps maps,
                                                                         const PairParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t stage_bytes = kABytes + p.b_bytes;
  const uint32_t staging = base + p.stages * stage_bytes;
  const uint32_t scales = staging + kEpilogueWarps * kPieces<kEpi> * kBoxBytes;
  const uint32_t bars = (scales + (kEpi == kScaled ? 2 * kEpilogueWarps * kScaleBytes : 0) + 7) & ~7u;
  const uint32_t bar_full = bars, bar_empty = bars + 8 * p.stages;
  const uint32_t bar_tfull = bar_empty + 8 * p.stages, bar_tempty = bar_tfull + 16, bar_in = bar_tempty + 16;
  const uint32_t slot = bar_in + 8 * kEpilogueWarps;
  volatile int* abort_p = reinterpret_cast<volatile int*>(smem_raw + (slot + 4 - smem_u32(smem_raw)));

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int tiles = p.tiles_m * p.tiles_n * p.splits;

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
  cluster_sync_all();  // both CTAs' barriers are initialised
  tc_fence_after();
  uint32_t tmem;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));

  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (p.more) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // 8-bit: the epilogue's sums take registers that the other warps do not need (128 x 80 + 256 x 208 of
  // the 384 x 168 that the block starts with)
  if (warp < 4) {
    if constexpr (kEightBit<kEpi>) asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 0) {
      if (elect_one()) {
        uint32_t s = 0, ph = 0;
        const uint32_t full0 = cluster_map_shared(bar_full, 0);
        const int box_b = int(p.b_bytes) / 8192;
        bool ok = true;
        for (int t = pair; ok && t < tiles; t += pairs) {
          const Tile tl = tile_of(p, t);
          const bool second = tl.m >= p.tiles_m0;
          const int m0 = (second ? tl.m - p.tiles_m0 : tl.m) * 256 + int(rank) * 128;
          const int n0 = p.paired ? tl.n * 128 : tl.n * p.block_n + int(rank) * (p.block_n >> 1);
          const int k0 = tl.split * p.kb_split, k1 = min(p.kb_total, k0 + p.kb_split);
          for (int kb = k0; kb < k1; ++kb) {
            if (!mbar_wait(bar_empty + 8 * s, ph ^ 1, abort_p, p.status, kStatProducerWait, p.limit_ns)) {
              ok = false;
              break;
            }
            const bool seg = kb >= p.kb_seg;
            const int k = (seg ? kb - p.kb_seg : kb) * (kEightBit<kEpi> ? 128 : 64);
            const CUtensorMap* ma = &maps.a[seg || second];
            const CUtensorMap* mb = &maps.b[seg || (p.paired && rank)];
            const uint32_t a = base + s * stage_bytes, b = a + kABytes, bar = full0 + 8 * s;
            if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * s, 2 * stage_bytes);
            if (p.a_kmajor) {
              tma_load_2d_pair(a, ma, k, m0, bar);
            } else {
              tma_load_2d_pair(a, ma, m0, k, bar);
              tma_load_2d_pair(a + 8192, ma, m0 + 64, k, bar);
            }
            if (p.b_kmajor) {
              tma_load_2d_pair(b, mb, k, n0, bar);
            } else {
              for (int i = 0; i < box_b; ++i) tma_load_2d_pair(b + 8192 * i, mb, n0 + 64 * i, k, bar);
            }
            if (++s == uint32_t(p.stages)) s = 0, ph ^= 1;
          }
        }
      }
    } else if (warp == 1) {
      if (rank == 0) {
        const bool issue = elect_one();
        uint32_t s = 0, ph = 0, buf = 0, bph = 0;
        bool ok = true;
        for (int t = pair; ok && t < tiles; t += pairs) {
          const Tile tl = tile_of(p, t);
          const int k0 = tl.split * p.kb_split, k1 = min(p.kb_total, k0 + p.kb_split);
          if constexpr (!kEightBit<kEpi>) {
            if (!wait_all(bar_tempty + 8 * buf, bph ^ 1, abort_p, p.status, kStatMmaWaitTmem, p.limit_ns)) break;
            tc_fence_after();
          }
          for (int kb = k0; kb < k1; ++kb) {
            if constexpr (kEightBit<kEpi>) {  // sums of one block of 128 a time
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
            const uint32_t a = base + s * stage_bytes;
            if (issue) {
              const uint64_t da = p.a_desc + (a >> 4), db = p.b_desc + ((a + kABytes) >> 4);
  #pragma unroll
              for (int j = 0; j < 4; ++j) {
                if constexpr (kEightBit<kEpi>) pair_mma_f8(d, da + j * 2, db + j * 2, p.idesc, j > 0);
                else pair_mma_f16(d, da + j * p.a_step, db + j * p.b_step, p.idesc, kb > k0 || j > 0);
              }
              pair_commit(bar_empty + 8 * s);
              if constexpr (kEightBit<kEpi>) pair_commit(bar_tfull + 8 * buf);
            }
            __syncwarp();
            if constexpr (kEightBit<kEpi>) {
              if (++buf == 2) buf = 0, bph ^= 1;
            }
            if (++s == uint32_t(p.stages)) s = 0, ph ^= 1;
          }
          if constexpr (!kEightBit<kEpi>) {
            if (issue && ok) pair_commit(bar_tfull + 8 * buf);
            __syncwarp();
            if (++buf == 2) buf = 0, bph ^= 1;
          }
        }
      }
    }
  } else {
    if constexpr (kEightBit<kEpi>) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int q = warp & 3, half = (warp - 4) >> 2;
    const uint32_t mine = staging + (warp - 4) * kPieces<kEpi> * kBoxBytes;
    const uint32_t in_bar = bar_in + 8 * (warp - 4);
    const uint32_t tempty0 = cluster_map_shared(bar_tempty, 0);
    const uint32_t lanes = tmem + (uint32_t(q * 32) << 16);
    uint32_t buf = 0, bph = 0, in_ph = 0, piece = 0;
    // The scales of 16 blocks of k from kb on, of tile t, on their way to half `b` of this warp's table.
    const uint32_t my_scales = scales + (warp - 4) * 2 * kScaleBytes;
    uint32_t sbuf = 0;
    auto fetch_scales = [&](const Tile& tl, int kb, uint32_t b) {
      const int sub = lane >> 4, k = min(kb + (lane & 15), p.kb_total - 1);
      const int64_t r0 = int64_t(tl.m) * 256 + int(rank) * 128 + q * 32 + sub;
      const int rows = int(min(int64_t(32), p.M - r0));  // from r0 on; what lies past them reads as 0
      const float* from = p.row_scale + min(r0, p.M - 1) * p.row_rs + k * p.row_ks;
      uint32_t to = my_scales + b * kScaleBytes + (lane & 15) * 4 + sub * 68;
#pragma unroll
      for (int r = 0; r < 32; r += 2) {
        cp_async4(to + r * 68, from, r < rows);
        if (r + 2 < rows) from += 2 * p.row_rs;
      }
      const int64_t nb = min((int64_t(tl.n) * p.block_n + half * (p.block_n >> 1)) >> 7, (p.N - 1) >> 7);
      if (sub == 0) cp_async4(to + 32 * 68, p.col_scale + nb * p.col_rs + k * p.col_ks, true);
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    Tile next = tile_of(p, pair);
    if constexpr (kEpi == kScaled) fetch_scales(next, 0, 0);
    for (int t = pair; t < tiles; t += pairs) {
      const Tile tl = next;
      next = tile_of(p, min(t + pairs, tiles - 1));
      const bool second = tl.m >= p.tiles_m0;
      const int row0 = (second ? tl.m - p.tiles_m0 : tl.m) * 256 + int(rank) * 128 + q * 32;
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
      if constexpr (kEpi == kStore) {
        if (!wait_sums()) break;
        const int cols = p.block_n >> 1;
        for (int c = 0; c < cols; c += 64) {
          float f[32], g[32];
          load_sums(acc + half * cols + c, f);
          load_sums(acc + half * cols + c + 32, g);
          if (c + 64 >= cols) release_sums();
          const uint32_t to = mine + piece * kBoxBytes;
          if (lane == 0) bulk_wait_group_read<1>();
          __syncwarp();
          stage32<T>(to, lane, 0, f);
          stage32<T>(to, lane, 4, g);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            const int col = tl.n * p.block_n + half * cols + c;
            if (row0 < p.M && col < p.N) tma_store_2d(&maps.out[second], to, col, row0);
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
          float unused;
#pragma unroll
          for (int i = 0; i < 32; ++i) g[i] = activation<false>(p.act, g[i], unused) * u[i];
          stage32<T>(mine, lane, c * 4, g);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (row0 < p.M && col < p.N) {
            tma_store_2d(&maps.out[0], mine, col, row0);
            if (p.save) {
              tma_store_2d(&maps.out[1], mine + kBoxBytes, col, row0);
              tma_store_2d(&maps.out[2], mine + 2 * kBoxBytes, col, row0);
            }
          }
          bulk_commit_group();
        }
      } else if constexpr (kEpi == kGatedBackward) {
        const int cols = p.block_n >> 1;
        bool first = true, ok = true;
        for (int c = 0; c < cols; c += 64) {
          const int col = tl.n * p.block_n + half * cols + c;
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
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              float da;
              const float a = activation<true>(p.act, g[i], da);
              g[i] = d[i] * u[i] * da;
              d[i] = d[i] * a;
              u[i] = a * u[i];
            }
            stage32<T>(mine, lane, j * 4, g);
            stage32<T>(mine + kBoxBytes, lane, j * 4, d);
            stage32<T>(mine + 2 * kBoxBytes, lane, j * 4, u);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (row0 < p.M && col < p.N) {
              tma_store_2d(&maps.out[0], mine, col, row0);
              tma_store_2d(&maps.out[1], mine + kBoxBytes, col, row0);
              tma_store_2d(&maps.out[2], mine + 2 * kBoxBytes, col, row0);
            }
            bulk_commit_group();
          }
        }
        if (!ok) break;
      } else if constexpr (kEpi == kScaled) {
        // Each block's sums are scaled and added up in registers (a row of half the columns a thread),
        // beside the MMAs of the next block: 128 columns are 64 two-wide multiply-adds.
        const int cols = p.block_n >> 1;
        uint64_t sum[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) sum[i] = 0;
        auto scale_of = [&](int kb) {
          if ((kb & 15) == 0) {
            // this half of the table has come; the other is free, as every lane is past its last use
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
            const bool on = kb + 16 < p.kb_total;
            fetch_scales(on ? tl : next, on ? kb + 16 : 0, sbuf ^ 1);
            sbuf ^= 1;
          }
          const uint32_t at = my_scales + (sbuf ^ 1) * kScaleBytes + (kb & 15) * 4;
          return ld_shared_f32(at + lane * 68) * ld_shared_f32(at + 32 * 68);
        };
        bool ok = true;
        for (int kb = 0; kb < p.kb_total; ++kb) {
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
        constexpr int kWidth = 128 / int(sizeof(T));  // columns of a piece
#pragma unroll
        for (int c = 0; c < 128; c += kWidth) {
          if (c < cols) {
            const uint32_t to = mine;
            if (lane == 0) bulk_wait_group_read<0>();
            __syncwarp();
            float f[kWidth];
#pragma unroll
            for (int i = 0; i < kWidth / 2; ++i) {
              const float2 v = halves_of(sum[c / 2 + i]);
              f[2 * i] = v.x;
              f[2 * i + 1] = v.y;
            }
            if constexpr (sizeof(T) == 4) {
              stage_f32(to, lane, f);
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                st_shared_v4(chunk_at(to, lane, j), pack2<T>(f[8 * j], f[8 * j + 1]), pack2<T>(f[8 * j + 2], f[8 * j + 3]),
                             pack2<T>(f[8 * j + 4], f[8 * j + 5]), pack2<T>(f[8 * j + 6], f[8 * j + 7]));
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              const int col = tl.n * p.block_n + half * cols + c;
              if (row0 < p.M && col < p.N) tma_store_2d(&maps.out[0], to, col, row0);
              bulk_commit_group();
            }
          }
        }
        continue;  // the buffers were handed on block by block
      } else if constexpr (kEpi == kScaledPartial) {
        // As kPartial, of 8-bit operands: rows are features (128 of a CTA share a scale), columns tokens
        // (a scale each, held by one lane and passed round).
        const int cols = max(p.block_n >> 1, 32);
        const int k0 = tl.split * p.kb_split, k1 = min(p.kb_total, k0 + p.kb_split);
        const bool busy = half * cols < p.block_n;
        const int n = tl.n * p.block_n + half * cols;
        const int64_t mb = min(int64_t(row0) >> 7, (p.M - 1) >> 7);
        float2 sum[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) sum[i] = make_float2(0.0f, 0.0f);
        bool ok = true;
        for (int kb = k0; kb < k1; ++kb) {
          const float sb = p.row_scale[mb * p.row_rs + kb * p.row_ks];
          float sa[4];
#pragma unroll
          for (int c = 0; c < 4; ++c)
            sa[c] = c * 32 < cols ? sb * p.col_scale[min(int64_t(n + c * 32 + lane), p.N - 1) * p.col_rs + kb * p.col_ks] : 0.0f;
          if (!(ok = wait_sums())) break;
          if (busy) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if (c * 32 < cols) {
                float f[32];
                load_sums(acc + half * cols + c * 32, f);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  sum[c * 16 + i].x += f[2 * i] * __shfl_sync(0xffffffffu, sa[c], 2 * i);
                  sum[c * 16 + i].y += f[2 * i + 1] * __shfl_sync(0xffffffffu, sa[c], 2 * i + 1);
                }
              }
            }
          }
          release_sums();
          if (++buf == 2) buf = 0, bph ^= 1;
          acc = lanes + buf * 256;
        }
        if (!ok) break;
        float* to = p.partial + tl.split * p.slice + int64_t(tl.m) * 256 + rank * 128 + q * 32 + lane;
#pragma unroll
        for (int c = 0; c < 128; ++c)
          if (busy && c < cols && n + c < p.N) to[(n + c) * p.pitch] = c & 1 ? sum[c / 2].y : sum[c / 2].x;
        continue;
      } else {  // kPartial: lanes are neighbours along the table's rows; the table covers whole tiles
        if (!wait_sums()) break;
        const int cols = max(p.block_n >> 1, 32);
        float* to = p.partial + tl.split * p.slice + int64_t(tl.m) * 256 + rank * 128 + q * 32 + lane;
        if (half * cols < p.block_n) {
          for (int c = 0; c < cols; c += 32) {
            float f[32];
            load_sums(acc + half * cols + c, f);
            const int n = tl.n * p.block_n + half * cols + c;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (n + i < p.N) to[(n + i) * p.pitch] = f[i];
          }
        }
        release_sums();
      }
      if (++buf == 2) buf = 0, bph ^= 1;
    }
    if constexpr (kEpi == kScaled) asm volatile("cp.async.wait_all;" ::: "memory");
    if (kPieces<kEpi> > 0 && lane == 0) bulk_wait_group<0>();
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
  cluster_sync_all();  // nothing arrives at, or reads, the other CTA's shared memory any more
  tc_fence_after();
  if (warp == 2) pair_tmem_dealloc(tmem, kTmemCols);
}

template <int kEpi, typename T>
cudaError_t launch_pair(const PairMaps& maps, const PairParams& p, int sms, bool chained, cudaStream_t s) {
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
  const int tiles = p.tiles_m * p.tiles_n * p.splits;
  const int pairs = tiles < sms / 2 ? tiles : sms / 2;
  const size_t smem = 1024 + size_t(p.stages) * (kABytes + p.b_bytes) + kEpilogueWarps * staged_pieces(kEpi) * kBoxBytes +
                      scale_bytes(kEpi) + kBarrierBytes;
  return launch(f, dim3(unsigned(2 * pairs)), kThreads, smem, 2, chained, s, maps, p);
}

template <int kEpi>
cudaError_t launch_scaled(int dtype, const PairMaps& maps, const PairParams& p, int sms, bool chained, cudaStream_t s) {
  if (dtype == CCONV_TYPE_BF16) return launch_pair<kEpi, __nv_bfloat16>(maps, p, sms, chained, s);
  if (dtype == CCONV_TYPE_FP16) return launch_pair<kEpi, __half>(maps, p, sms, chained, s);
  return launch_pair<kEpi, float>(maps, p, sms, chained, s);
}

template <typename T>
cudaError_t launch_epilogue(int epi, const PairMaps& maps, const PairParams& p, int sms, bool chained, cudaStream_t s) {
  if (epi == kStore) return launch_pair<kStore, T>(maps, p, sms, chained, s);
  if (epi == kGated) return launch_pair<kGated, T>(maps, p, sms, chained, s);
  if (epi == kGatedBackward) return launch_pair<kGatedBackward, T>(maps, p, sms, chained, s);
  return launch_pair<kPartial, T>(maps, p, sms, chained, s);
}

int encode_operand(CUtensorMap* tm, const Operand& o, int es, int dtype, int rows_box) {
  if (es == 1) return encode_map(tm, o.p, 1, dtype, o.k, o.rows, o.pitch, 128, rows_box);
  return o.kmajor ? encode_map(tm, o.p, 2, dtype, o.k, o.rows, o.pitch, 64, rows_box)
                  : encode_map(tm, o.p, 2, dtype, o.rows, o.k, o.pitch, 64, 64);
}

// ---- finishing passes: four neighbouring columns a thread, a row a blockIdx.y step -----------------
__device__ __forceinline__ void add_up(const Partial& p, int64_t at, float (&f)[4]) {
  float4 v = *reinterpret_cast<const float4*>(p.p + at);
  for (int s = 1; s < p.splits; ++s) {
    const float4 w = *reinterpret_cast<const float4*>(p.p + s * p.slice + at);
    v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
  }
  f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
}
template <typename T>
__device__ __forceinline__ void put4(const Mat& m, int64_t r, int64_t c, int64_t N, const float (&f)[4]) {
  T* o = static_cast<T*>(const_cast<void*>(m.p)) + r * m.rs + c * m.cs;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < N) o[i * m.cs] = from_f32<T>(f[i]);
}
template <typename T>
__device__ __forceinline__ void get4(const Mat& m, int64_t r, int64_t c, int64_t N, float (&f)[4]) {
  const T* o = static_cast<const T*>(m.p) + r * m.rs + c * m.cs;
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = c + i < N ? to_f32(o[i * m.cs]) : 0.0f;
}
#define CCONV_FINISH_PROLOGUE                                                          \
  asm volatile("griddepcontrol.wait;" ::: "memory");                                   \
  if (more) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");            \
  const int64_t n = (int64_t(blockIdx.x) * 128 + threadIdx.x) * 4;                     \
  if (n >= N) return;

template <typename T>
__global__ void __launch_bounds__(128) finish_store_kernel(Partial p, Mat out, int64_t M, int64_t N, int more) {
  CCONV_FINISH_PROLOGUE
  for (int64_t m = blockIdx.y; m < M; m += gridDim.y) {
    float f[4];
    add_up(p, m * p.pitch + n, f);
    put4<T>(out, m, n, N, f);
  }
}

template <typename T>
__global__ void __launch_bounds__(128) finish_gated_kernel(Partial p, Mat gate_pre, Mat up_pre, Mat h, int64_t M,
                                                           int64_t N, int act, int more) {
  CCONV_FINISH_PROLOGUE
  for (int64_t m = blockIdx.y; m < M; m += gridDim.y) {
    float g[4], u[4], f[4], da;
    add_up(p, m * p.pitch + n, g);
    add_up(p, m * p.pitch + p.second + n, u);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = activation<false>(act, g[i], da) * u[i];
    put4<T>(h, m, n, N, f);
    if (gate_pre.p) {
      put4<T>(gate_pre, m, n, N, g);
      put4<T>(up_pre, m, n, N, u);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(128) finish_gated_backward_kernel(Partial p, Mat gate_pre, Mat up_pre, Mat dg,
                                                                    Mat du, Mat h, int64_t M, int64_t N, int act,
                                                                    int more) {
  CCONV_FINISH_PROLOGUE
  for (int64_t m = blockIdx.y; m < M; m += gridDim.y) {
    float d[4], g[4], u[4], f[4];
    get4<T>(gate_pre, m, n, N, g);
    get4<T>(up_pre, m, n, N, u);
    add_up(p, m * p.pitch + n, d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float da;
      const float a = activation<true>(act, g[i], da);
      g[i] = d[i] * u[i] * da;
      f[i] = d[i] * a;
      u[i] = a * u[i];
    }
    put4<T>(dg, m, n, N, g);
    put4<T>(du, m, n, N, f);
    put4<T>(h, m, n, N, u);
  }
}

// 32 x 32 elements a block through shared memory: read along the source's short stride, written along
// the target's.
template <typename E>
__global__ void __launch_bounds__(256) cconv_copy_kernel(Mat from, Mat to, int64_t rows, int64_t cols, int more) {
  __shared__ E tile[32][33];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (more) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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

dim3 finish_grid(int64_t M, int64_t N) { return dim3(unsigned(cdiv64(N, 512)), unsigned(M < 16384 ? M : 16384)); }

}  // namespace

uint64_t block_wait_limit_ns() {
  const char* v = std::getenv("CCONV_WAIT_LIMIT_MS");
  return uint64_t(v && *v ? std::atoi(v) : 1000) * 1000000ull;
}

int block_status_word(int** word) {
  void* p = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&p, g_block_status);
  *word = static_cast<int*>(p);
  return block_cuda_error(e, "cudaGetSymbolAddress");
}

int64_t partial_rows(int64_t M, int stack) { return cdiv64(M, 256) * 256 * stack; }

cudaError_t run_product(const Product& p, int sms, bool chained, bool more, cudaStream_t s, int* rc) {
  PairMaps maps;
  PairParams q{};
  *rc = block_status_word(&q.status);
  if (*rc) return cudaSuccess;
  const int stack = p.stacked ? 2 : 1;
  q.tiles_m0 = int(cdiv64(p.M, 256));
  q.tiles_m = q.tiles_m0 * stack;
  q.tiles_n = int(cdiv64(p.N, p.paired ? 128 : p.block_n));
  const bool eight = p.epilogue == kScaled || p.epilogue == kScaledPartial;
  q.kb_seg = int(cdiv64(p.K, eight ? 128 : 64));
  q.kb_total = q.kb_seg * (p.segments ? 2 : 1);
  q.kb_split = int(cdiv64(q.kb_total, p.splits));
  q.splits = int(cdiv64(q.kb_total, q.kb_split));
  q.block_n = p.block_n;
  q.b_bytes = uint32_t(p.block_n / 2) * 128;
  const uint32_t staged = kEpilogueWarps * staged_pieces(p.epilogue) * kBoxBytes + scale_bytes(p.epilogue);
  q.stages = int((kSmemMost - 1024 - kBarrierBytes - staged) / (kABytes + q.b_bytes));
  if (q.stages > 8) q.stages = 8;
  q.a_kmajor = p.a[0].kmajor;
  q.b_kmajor = p.b[0].kmajor;
  q.paired = p.paired;
  q.a_desc = swizzled_desc(p.a[0].kmajor, 8192);
  q.b_desc = swizzled_desc(p.b[0].kmajor, 8192);
  q.a_step = p.a[0].kmajor ? 32 >> 4 : 2048 >> 4;
  q.b_step = p.b[0].kmajor ? 32 >> 4 : 2048 >> 4;
  const uint32_t type = !eight && p.dtype == CCONV_TYPE_BF16 ? 1u : 0u;  // (8 bits: 0 is e4m3)
  // instruction descriptor: D fp32, types of A and B, their orders (1: rows contiguous), N / 8, M / 16
  q.idesc = (1u << 4) | (type << 7) | (type << 10) | (uint32_t(!p.a[0].kmajor) << 15) |
            (uint32_t(!p.b[0].kmajor) << 16) | (uint32_t(p.block_n >> 3) << 17) | (uint32_t(256 >> 4) << 24);
  q.M = p.M;
  q.N = p.N;
  q.act = p.act;
  q.save = p.save;
  q.more = more;
  q.partial = p.partial;
  q.pitch = p.pitch;
  q.slice = p.slice;
  q.row_scale = static_cast<const float*>(p.row_scale.p);
  q.row_rs = p.row_scale.rs;
  q.row_ks = p.row_scale.cs;
  q.col_scale = static_cast<const float*>(p.col_scale.p);
  q.col_rs = p.col_scale.rs;
  q.col_ks = p.col_scale.cs;
  q.limit_ns = block_wait_limit_ns();
  const int two_a = p.segments || p.stacked ? 2 : 1, two_b = p.segments || p.paired ? 2 : 1;
  for (int i = 0; i < 2; ++i) {
    if ((*rc = encode_operand(&maps.a[i], p.a[i < two_a ? i : 0], eight ? 1 : 2, p.dtype, 128))) return cudaSuccess;
    if ((*rc = encode_operand(&maps.b[i], p.b[i < two_b ? i : 0], eight ? 1 : 2, p.dtype, p.block_n / 2))) return cudaSuccess;
  }
  for (int i = 0; i < 5; ++i) {
    const Mat& m = i < 3 ? p.out[i] : p.in[i - 3];
    CUtensorMap* tm = i < 3 ? &maps.out[i] : &maps.in[i - 3];
    *tm = maps.a[0];
    if (m.p && (*rc = encode_map(tm, m.p, type_bytes(p.dtype), p.dtype, p.N, p.M, m.rs, 128 / type_bytes(p.dtype), 32))) return cudaSuccess;
  }
  if (p.epilogue == kScaled) return launch_scaled<kScaled>(p.dtype, maps, q, sms, chained, s);
  if (p.epilogue == kScaledPartial) return launch_pair<kScaledPartial, float>(maps, q, sms, chained, s);
  return p.dtype == CCONV_TYPE_BF16 ? launch_epilogue<__nv_bfloat16>(p.epilogue, maps, q, sms, chained, s)
                                    : launch_epilogue<__half>(p.epilogue, maps, q, sms, chained, s);
}

cudaError_t finish_store(const Partial& p, const Mat& out, int64_t M, int64_t N, int dtype, bool more, cudaStream_t s) {
  auto f = dtype == CCONV_TYPE_BF16   ? finish_store_kernel<__nv_bfloat16>
           : dtype == CCONV_TYPE_FP16 ? finish_store_kernel<__half>
                                      : finish_store_kernel<float>;
  return launch(f, finish_grid(M, N), 128, 0, 1, true, s, p, out, M, N, int(more));
}

cudaError_t finish_gated(const Partial& p, const Mat& gate_pre, const Mat& up_pre, const Mat& h, int64_t M, int64_t N,
                         int act, int dtype, bool more, cudaStream_t s) {
  auto f = dtype == CCONV_TYPE_BF16 ? finish_gated_kernel<__nv_bfloat16> : finish_gated_kernel<__half>;
  return launch(f, finish_grid(M, N), 128, 0, 1, true, s, p, gate_pre, up_pre, h, M, N, act, int(more));
}

cudaError_t finish_gated_backward(const Partial& p, const Mat& gate_pre, const Mat& up_pre, const Mat& dg,
                                  const Mat& du, const Mat& h, int64_t M, int64_t N, int act, int dtype, bool more,
                                  cudaStream_t s) {
  auto f = dtype == CCONV_TYPE_BF16 ? finish_gated_backward_kernel<__nv_bfloat16> : finish_gated_backward_kernel<__half>;
  return launch(f, finish_grid(M, N), 128, 0, 1, true, s, p, gate_pre, up_pre, dg, du, h, M, N, act, int(more));
}

cudaError_t run_copy(const Mat& from, const Mat& to, int64_t rows, int64_t cols, int es, bool chained, bool more,
                     cudaStream_t s) {
  if (rows == 0 || cols == 0) return cudaSuccess;
  const int64_t y = cdiv64(rows, 32);
  const dim3 grid(unsigned(cdiv64(cols, 32)), unsigned(y < 65535 ? y : 65535));
  if (es == 1) return launch(cconv_copy_kernel<uint8_t>, grid, 256, 0, 1, chained, s, from, to, rows, cols, int(more));
  if (es == 4) return launch(cconv_copy_kernel<uint32_t>, grid, 256, 0, 1, chained, s, from, to, rows, cols, int(more));
  return launch(cconv_copy_kernel<uint16_t>, grid, 256, 0, 1, chained, s, from, to, rows, cols, int(more));
}

}  // namespace cconv
