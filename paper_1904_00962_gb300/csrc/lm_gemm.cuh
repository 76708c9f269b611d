// Matrix products of the language-model operators: C = A B^T of bf16 or fp16
// operands with fp32 accumulators, tile by tile, each tile handed to an
// epilogue while the next one is multiplied.
//
// One persistent CTA per SM walks the tiles of a Work type:
//   Work::kBf16                   operands bf16 (else fp16)
//   Work::Params::status          the plan's status word
//   Work::start(params)           what the kernel reads first: State, with the
//                                 number of tiles (it may come from the device)
//   Work::tile(params, state, t)  operands and extent of tile t (GemmTile)
//   Work::epilogue(params, state, tile, acc, epi)  a row of the accumulator
// A tile is 128 rows of A by 256 of B.  Operands come through tensor maps with
// the 128-byte swizzle, K-major (64 of K by all the tile's rows) or MN-major
// (blocks of 64 rows by 64 of K, all of the tile's in one copy where the map has
// them as a third dimension); what lies outside a matrix arrives as zeros.  One
// copy an operand counts: issuing one takes its thread some 100 cycles, and a
// stage of products 512.
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
constexpr int kTileBytesB = kTileN * kTileK * 2;
constexpr int kGemmStageBytes = kTileBytesA + kTileBytesB;
constexpr int kGemmStages = 4;
// a block of 32 rows and 64 columns on its way out, two a warp
constexpr int kOutBytes = 32 * 64 * 2, kOutBuffers = 2;
constexpr size_t kGemmSmem = (size_t)kGemmStages * kGemmStageBytes +
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
  uint64_t full[kGemmStages], empty[kGemmStages];
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem;
  volatile int gave_up;
};

// What an epilogue thread has.
struct Epilogue {
  int row;               // of the tile, 0 .. 127
  uint32_t out;          // the warp's staging memory
  int n;                 // blocks that went through it

  // A block of the warp's 32 rows and 64 columns of 16 bits, w the thread's row:
  // out by a tensor copy to (x, y), which clips it at the matrix' edges.  Direct
  // stores, a row a thread, take a 16-byte piece of 32 lines each.
  __device__ __forceinline__ void store_block(const CUtensorMap* map, int x,
                                              int y, const uint32_t (&w)[32]) {
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
      tile_store(map, x, y, at);
      stores_commit();
    }
    ++n;
  }

  // Every thread, whatever its wait said: one answer for all.
  __device__ __forceinline__ bool all(bool x) const {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, %2, %3, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r) : "r"((uint32_t)x), "n"(kEpiBarrier), "n"(kEpiThreads)
        : "memory");
    return r != 0;
  }
};

template <class Work>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_kernel(const __grid_constant__ typename Work::Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ GemmShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem =
      (smem_u32(smem_raw) + 1023u) & ~1023u;   // the swizzle's pattern

  if (threadIdx.x == 0) {
    for (int i = 0; i < kGemmStages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.acc_full[i], 1);
      mbar_init(&sh.acc_empty[i], 4);
    }
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  if (warp == 2) tmem_alloc_all(&sh.tmem);
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  const uint32_t tmem = sh.tmem;
  let_next_launch();
  after_prior_launch();
  const typename Work::State st = Work::start(p);

  if (warp == 0) {
    if (elect_lane()) {
      int it = 0;
      bool ok = true;
      for (int t = blockIdx.x; ok && t < st.n_tiles; t += gridDim.x) {
        const GemmTile g = Work::tile(p, st, t);
        for (int kb = 0; kb < g.kn; ++kb, ++it) {
          const int s = it % kGemmStages;
          const uint32_t ph = (uint32_t)(it / kGemmStages) & 1u;
          if (!bounded_wait(&sh.empty[s], ph ^ 1u, &sh.gave_up, p.status,
                            kStatusWaitTimeout)) {
            ok = false;
            break;
          }
          const uint32_t at = smem + s * kGemmStageBytes;
          const int k = (g.k0 + kb) * kTileK;
          mbar_expect(&sh.full[s], kGemmStageBytes);
          if (g.a_mn) blocks_load(at, g.a, k, g.a0 / 64, &sh.full[s]);
          else tile_load(at, g.a, k, g.a0, &sh.full[s]);
          const uint32_t bt = at + kTileBytesA;
          const int bk = k + g.b_k;
          if (!g.b_mn) {
            tile_load(bt, g.b, bk, g.b0, &sh.full[s]);
          } else if (g.b_blocks) {
            blocks_load(bt, g.b, bk, g.b0 / 64, &sh.full[s]);
          } else {
            for (int i = 0; i < 4; ++i)
              tile_load(bt + i * 8192, g.b, g.b0 + 64 * i, bk, &sh.full[s]);
          }
        }
      }
      // every copy has landed, and its products' arrival is in, before the CTA
      // may leave
      const int first = it > kGemmStages ? it - kGemmStages : 0;
      for (int j = first; j < it; ++j) {
        settle(&sh.full[j % kGemmStages], (uint32_t)(j / kGemmStages) & 1u);
        bounded_wait(&sh.empty[j % kGemmStages],
                     (uint32_t)(j / kGemmStages) & 1u, &sh.gave_up, p.status,
                     kStatusWaitTimeout);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (elect_lane()) {
      int it = 0, n = 0;
      bool ok = true;
      for (int t = blockIdx.x; ok && t < st.n_tiles; t += gridDim.x, ++n) {
        const GemmTile g = Work::tile(p, st, t);
        const uint64_t da = operand_desc(g.a_mn), db = operand_desc(g.b_mn);
        const uint32_t sa = operand_step(g.a_mn), sb = operand_step(g.b_mn);
        const uint32_t desc =
            product_desc(Work::kBf16, g.a_mn, g.b_mn, kTileM, kTileN);
        const int acc = n & 1;
        const uint32_t d = tmem + acc * kTileN;
        if (!bounded_wait(&sh.acc_empty[acc], ((uint32_t)(n >> 1) & 1u) ^ 1u,
                          &sh.gave_up, p.status, kStatusWaitTimeout))
          break;
        tmem_after_sync();
        for (int kb = 0; kb < g.kn; ++kb, ++it) {
          const int s = it % kGemmStages;
          if (!bounded_wait(&sh.full[s], (uint32_t)(it / kGemmStages) & 1u,
                            &sh.gave_up, p.status, kStatusWaitTimeout)) {
            ok = false;
            break;
          }
          tmem_after_sync();
          const uint32_t at = smem + s * kGemmStageBytes;
          const uint64_t a = da | (at >> 4), b = db | ((at + kTileBytesA) >> 4);
#pragma unroll
          for (int k = 0; k < kTileK / 16; ++k)
            product(d, a + k * sa, b + k * sb, desc, kb > 0 || k > 0);
          products_arrive(&sh.empty[s]);
        }
        if (ok) products_arrive(&sh.acc_full[acc]);
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    Epilogue epi;
    const int quarter = warp & 3;
    epi.row = quarter * 32 + lane;
    epi.out = smem + kGemmStages * kGemmStageBytes +
              quarter * (kOutBuffers * kOutBytes);
    epi.n = 0;
    int n = 0;
    for (int t = blockIdx.x; t < st.n_tiles; t += gridDim.x, ++n) {
      const GemmTile g = Work::tile(p, st, t);
      const int acc = n & 1;
      const bool ok =
          bounded_wait(&sh.acc_full[acc], (uint32_t)(n >> 1) & 1u, &sh.gave_up,
                       p.status, kStatusWaitTimeout);
      if (!epi.all(ok)) break;
      tmem_after_sync();
      Work::epilogue(p, st, g,
                     tmem + acc * kTileN + ((uint32_t)(quarter * 32) << 16),
                     epi);
      tmem_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.acc_empty[acc]);
    }
    if (lane == 0) stores_done();
  }
  tmem_before_sync();
  __syncthreads();
  tmem_after_sync();
  if (warp == 2) tmem_free_all(tmem);
}

}  // namespace
}  // namespace lamb
