// Matrix products of the language-model operators: C = A B^T of bf16 or fp16
// operands with fp32 accumulators, tile by tile, each tile handed to an
// epilogue while the next one is multiplied.
//
// Persistent CTAs walk the tiles of a Work type, one by one or in pairs (kCtas): a
// pair multiplies a tile of 256 x 256 (cta_group::2), each CTA holding 128 rows of
// A and of B.  A pair's stage takes two thirds of what two single ones do, so six
// fit instead of four and less comes from L2; a single CTA's tile of 128 rows wastes
// less on few rows.
//   Work::kBf16                   operands bf16 (else fp16)
//   Work::Params::status          the plan's status word
//   Work::start<kRows>(params)    what the kernel reads first: State (numbers of
//                                 tiles of kRows rows may come from the device)
//   Work::tile<kRows>(params, state, u, units, i, tile)   operands and extent
//                                 (GemmTile) of the i-th tile of CTA or pair u;
//                                 false past its last
//   Work::early(params, u, tile)  whether the first tile of CTA u is known, and its
//                                 B there, before the launch in front has ended
//   Work::epilogue(params, state, tile, acc, epi)  a row of the accumulator
// A tile has 256 rows of B.  Operands come through tensor maps with the 128-byte
// swizzle, K-major (64 of K by all of a CTA's rows) or MN-major (blocks of 64 rows
// by 64 of K, all of a CTA's in one copy where the map has them as a third
// dimension); what lies outside a matrix arrives as zeros.  One copy an operand
// counts: issuing one takes its thread some 100 cycles, and a stage of products
// 512.
//
// Warps: 0 copies, 1 issues the products, 2 holds the tensor memory, 4-7 run the
// epilogue (a warp reaches the quarter of the lanes with its number mod 4).
// Two accumulators of 256 columns fill tensor memory, so a tile's epilogue runs
// beside the next tile's products.
#pragma once
#include "lamb_internal.h"
#include "lm_tc.cuh"

namespace lamb {
namespace {

constexpr int kTileM = 128, kTileN = 256, kTileK = 64;
constexpr int kGemmThreads = 256;
constexpr int kTileBytesA = kTileM * kTileK * 2;
// a CTA's rows of B, stages
template <int kCtas>
constexpr int kRowsB = kTileN / kCtas;
template <int kCtas>
constexpr int kGemmStageBytes = kTileBytesA + kRowsB<kCtas> * kTileK * 2;
template <int kCtas>
constexpr int kGemmStages = kCtas == 2 ? 6 : 4;
constexpr int kMaxStages = 6;
// a block of 32 rows and 64 columns on its way out, two a warp
constexpr int kOutBytes = 32 * 64 * 2, kOutBuffers = 2;
template <int kCtas>
constexpr size_t kGemmSmem =
    (size_t)kGemmStages<kCtas> * kGemmStageBytes<kCtas> +
    4 * kOutBuffers * kOutBytes + 1024;
constexpr int kEpiThreads = 128, kEpiBarrier = 1;

struct GemmTile {
  const CUtensorMap* a;
  const CUtensorMap* b;
  int a0, b0;        // first row of A, of B
  int k0, kn;        // first block of K, number of blocks
  int b_k;           // elements that B's K starts further on
  bool a_mn, b_mn;   // MN-major operands
  bool b_blocks;     // B's blocks are a dimension of its map (A's always are)
  int what, aux;     // the epilogue's
};

struct GemmShared {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem;
  volatile int gave_up;
};

// What an epilogue thread has.
struct Epilogue {
  int row;               // of the tile, 0 .. 127
  uint32_t out;          // the warp's staging memory
  int n;                 // blocks that went through it

  // A block of the warp's 32 rows and 128 bytes of columns, w the thread's row:
  // out by a tensor copy to (x, y), which clips it at the matrix' edges, or added
  // to what is there (fp32).  Direct stores, a row a thread, take a 16-byte piece
  // of 32 lines each.
  __device__ __forceinline__ void store_block(const CUtensorMap* map, int x,
                                              int y, const uint32_t (&w)[32],
                                              bool add = false) {
    const int r = row & 31;
    const uint32_t at = out + (n & 1) * kOutBytes;
    if (r == 0) stores_have_read<kOutBuffers - 1>();
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q)
      sts16(at + r * 128 + ((q ^ (r & 7)) << 4),
            make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]));
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (r == 0) {
      if (add) tile_add(map, x, y, at);
      else tile_store(map, x, y, at);
      stores_commit();
    }
    ++n;
  }
};

template <class Work, int kCtas>
__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kGemmThreads, 1)
gemm_kernel(const __grid_constant__ typename Work::Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ GemmShared sh;
  constexpr bool kPair = kCtas == 2;
  constexpr int kStages = kGemmStages<kCtas>, kRows = kTileM * kCtas;
  constexpr uint32_t kBytes = kGemmStageBytes<kCtas>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem =
      (smem_u32(smem_raw) + 1023u) & ~1023u;   // the swizzle's pattern
  const int rank = kPair ? (int)cluster_rank() : 0;
  const int unit = blockIdx.x / kCtas, units = gridDim.x / kCtas;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.acc_full[i], 1);
      mbar_init(&sh.acc_empty[i], 4 * kCtas);
    }
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  if (warp == 2) {
    if (kPair) pair_tmem_alloc_all(&sh.tmem);
    else tmem_alloc_all(&sh.tmem);
  }
  tmem_before_sync();
  __syncthreads();
  if (kPair) cluster_sync();
  tmem_after_sync();
  const uint32_t tmem = sh.tmem;
  let_next_launch();
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    return bounded_wait(bar, parity, &sh.gave_up, p.status, kStatusWaitTimeout);
  };

  if (warp == 0) {
    if (elect_lane()) {
      int it = 0, ahead = 0;       // ahead: blocks of B that are on their way
      bool ok = true;
      GemmTile e;
      if (!kPair && Work::early(p, unit, &e)) {
        for (; ahead < kStages && ahead < e.kn; ++ahead) {
          mbar_expect(&sh.full[ahead], kBytes);
          tile_load(smem + ahead * kBytes + kTileBytesA, e.b, ahead * kTileK,
                    e.b0, &sh.full[ahead]);
        }
      }
      after_prior_launch();
      const typename Work::State st = Work::template start<kRows>(p);
      GemmTile g;
      for (int i = 0;
           ok && Work::template tile<kRows>(p, st, unit, units, i, &g); ++i) {
        const int a0 = g.a0 + rank * kTileM;
        const int b0 = g.b0 + rank * kRowsB<kCtas>;
        for (int kb = 0; kb < g.kn; ++kb, ++it) {
          const int s = it % kStages;
          if (!wait(&sh.empty[s], ((uint32_t)(it / kStages) & 1u) ^ 1u)) {
            ok = false;
            break;
          }
          const uint32_t at = smem + s * kBytes, bt = at + kTileBytesA;
          const int k = (g.k0 + kb) * kTileK, bk = k + g.b_k;
          if (it < ahead) {
            tile_load(at, g.a, k, a0, &sh.full[s]);
            continue;
          }
          if (rank == 0) mbar_expect(&sh.full[s], kCtas * kBytes);
          if (kPair) {
            const uint32_t bar = at_rank(&sh.full[s], 0);   // who issues
            if (g.a_mn) pair_blocks_load(at, g.a, k, a0 / 64, bar);
            else pair_tile_load(at, g.a, k, a0, bar);
            if (!g.b_mn) {
              pair_tile_load(bt, g.b, bk, b0, bar);
            } else if (g.b_blocks) {
              pair_blocks_load(bt, g.b, bk, b0 / 64, bar);
            } else {
              for (int i = 0; i < kRowsB<kCtas> / 64; ++i)
                pair_tile_load(bt + i * 8192, g.b, b0 + 64 * i, bk, bar);
            }
          } else {
            if (g.a_mn) blocks_load(at, g.a, k, a0 / 64, &sh.full[s]);
            else tile_load(at, g.a, k, a0, &sh.full[s]);
            if (!g.b_mn) {
              tile_load(bt, g.b, bk, b0, &sh.full[s]);
            } else if (g.b_blocks) {
              blocks_load(bt, g.b, bk, b0 / 64, &sh.full[s]);
            } else {
              for (int i = 0; i < kRowsB<kCtas> / 64; ++i)
                tile_load(bt + i * 8192, g.b, b0 + 64 * i, bk, &sh.full[s]);
            }
          }
        }
      }
      // every copy has landed, and its products' arrival is in, before the CTA
      // (either of a pair: cluster_sync) may leave
      for (int j = it > kStages ? it - kStages : 0; j < it; ++j) {
        if (rank == 0 && sh.gave_up)
          settle(&sh.full[j % kStages], (uint32_t)(j / kStages) & 1u);
        wait(&sh.empty[j % kStages], (uint32_t)(j / kStages) & 1u);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && elect_lane()) {
      int it = 0, n = 0;
      bool ok = true;
      after_prior_launch();
      const typename Work::State st = Work::template start<kRows>(p);
      GemmTile g;
      for (; ok && Work::template tile<kRows>(p, st, unit, units, n, &g); ++n) {
        const uint64_t da = operand_desc(g.a_mn), db = operand_desc(g.b_mn);
        const uint32_t sa = operand_step(g.a_mn), sb = operand_step(g.b_mn);
        const uint32_t desc =
            product_desc(Work::kBf16, g.a_mn, g.b_mn, kRows, kTileN);
        const int acc = n & 1;
        const uint32_t d = tmem + acc * kTileN;
        const uint32_t ph = ((uint32_t)(n >> 1) & 1u) ^ 1u;
        if (!wait(&sh.acc_empty[acc], ph)) break;
        if (kPair) mbar_try_cluster(&sh.acc_empty[acc], ph);
        tmem_after_sync();
        for (int kb = 0; kb < g.kn; ++kb, ++it) {
          const int s = it % kStages;
          if (!wait(&sh.full[s], (uint32_t)(it / kStages) & 1u)) {
            ok = false;
            break;
          }
          tmem_after_sync();
          const uint32_t at = smem + s * kBytes;
          const uint64_t a = da | (at >> 4), b = db | ((at + kTileBytesA) >> 4);
#pragma unroll
          for (int k = 0; k < kTileK / 16; ++k) {
            if (kPair)
              pair_product(d, a + k * sa, b + k * sb, desc, kb > 0 || k > 0);
            else
              product(d, a + k * sa, b + k * sb, desc, kb > 0 || k > 0);
          }
          if (kPair) pair_products_arrive(&sh.empty[s]);
          else products_arrive(&sh.empty[s]);
        }
        if (ok) {
          if (kPair) pair_products_arrive(&sh.acc_full[acc]);
          else products_arrive(&sh.acc_full[acc]);
        }
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    after_prior_launch();
    const typename Work::State st = Work::template start<kRows>(p);
    Epilogue epi;
    const int quarter = warp & 3;
    epi.row = quarter * 32 + lane;
    epi.out = smem + kStages * kBytes + quarter * (kOutBuffers * kOutBytes);
    epi.n = 0;
    int n = 0;
    GemmTile g;
    for (; Work::template tile<kRows>(p, st, unit, units, n, &g); ++n) {
      g.a0 += rank * kTileM;
      const int acc = n & 1;
      const bool ok = wait(&sh.acc_full[acc], (uint32_t)(n >> 1) & 1u);
      if (!__all_sync(0xffffffffu, ok)) break;
      tmem_after_sync();
      Work::epilogue(p, st, g,
                     tmem + acc * kTileN + ((uint32_t)(quarter * 32) << 16),
                     epi);
      tmem_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (kPair) remote_arrive(at_rank(&sh.acc_empty[acc], 0));
        else mbar_arrive(&sh.acc_empty[acc]);
      }
    }
    if (lane == 0) stores_done();
  }
  tmem_before_sync();
  __syncthreads();
  if (kPair) cluster_sync();
  tmem_after_sync();
  if (warp == 2) {
    if (kPair) pair_tmem_free_all(tmem);
    else tmem_free_all(tmem);
  }
}

}  // namespace
}  // namespace lamb
