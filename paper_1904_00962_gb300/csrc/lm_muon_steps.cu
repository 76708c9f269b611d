// The products of the Muon update: all steps of all matrices in one launch.
//
// Per matrix and step: G = X X^T, G G, and (b G + c G G) X (lm_muon.cu has the
// splitting of G and X that keeps their precision).  A tile is 256 x 256 of one
// product, multiplied by a pair of CTAs (cta_group::2), 128 rows each, which copies
// an operand block to one of them only; or, where that makes too few tiles, 128 x
// 128 by one CTA.  A CTA's stage takes 32 KB either way, and four of them fit beside
// the epilogue's buffers.  The symmetric products' tiles are taken on and above the
// diagonal only.
//
// Persistent CTAs or pairs, one CTA an SM, take the tiles of one list in turn.  Two
// sets of matrices go through their steps side by side in it, so that while the last
// tiles of one set's product are still in work the other set's fill the SMs.  A tile
// of a product waits for all tiles of the product before it of the same matrix (a
// counter for each matrix).  Those come earlier in the list, which everybody takes
// in order, so the earliest unfinished tile waits for nothing; all CTAs are resident
// (cooperative launch).  Waits are bounded.
//
// Warps: 0 lists tiles and copies operands, 1 issues the products, 2 copies the
// epilogue's blocks in (and holds the tensor memory), 3 copies them out, 4-7 and
// 8-11 run the epilogue, every other block each.  A block is 32 columns of the
// tile: its inputs (X as hi and lo; D) come to a ring of staging buffers ahead of
// the products' end, the epilogue turns them over in place, a row a thread, and
// tensor copies take them out (clipped at the matrix' edges).  The tile is counted
// as done when those have landed.  Warp 0 reads the list a tile ahead and leaves in
// shared memory all that the other warps need of a tile.
//
// Measured: one 1024 x 1024 matrix 139 us with the momentum's launches, 15 products
// one behind another; one BERT-large layer (four 1024 x 1024, two 4096 x 1024) 308
// us, bound by the chain of a matrix' products (64 blocks of K, the epilogue's drain,
// the counters); all matrices of BERT-base 1355 us: X, D and E do not fit L2 and pass
// DRAM every step, 6.5 GB in all at 4.8 TB/s (61% of its peak, 0.71 of a copy's rate),
// the tensor pipe 43% busy.  Sets that do fit (56 MB each) wait for one another's
// products instead: 1500 us.  On the way there (both cases, us, with the momentum's
// launches): a launch a product with a CTA a tile 550 / 2909, one launch 419 / 2336,
// all matrices in two sets 419 / 1812, pairs of CTAs 353 / 1683.  X in fp32 beside hi
// in place of lo: 411 / 1963.
#include <algorithm>

#include "lm_gemm.cuh"
#include "lm_muon.h"

namespace lamb {
namespace {

constexpr int kStages = 4;
constexpr int kStageBytes = 2 * kTileBytesA;      // a CTA's rows of A and of B
constexpr int kBuffers = 5;
constexpr int kBlockBytes = kTileM * kMuonCols * 2;     // of one fp16 matrix
constexpr int kBufferBytes = 2 * kBlockBytes;
constexpr int kRing = 4;                                // tiles listed ahead
constexpr int kGroups = 2;                              // of epilogue warps
constexpr int kStepThreads = 128 + kGroups * kEpiThreads;
// readers of a listed tile: products, copies in, copies out, epilogue
constexpr int kReaders = 3 + 4 * kGroups;
// l or beta of a tile's columns, and of its rows
constexpr int kColBytes = 2 * kTileM * 4, kVecBytes = kColBytes + kTileM * 4;
constexpr size_t kSmem = (size_t)kStages * kStageBytes +
                         kBuffers * kBufferBytes + kRing * kVecBytes + 1024;
static_assert(kTileM == kMuonRows, "tiles");
// a tile's rows and columns: of one CTA, of a pair
template <int kCtas>
constexpr int kTile = kTileM * kCtas;

struct Listed : MuonTile {
  int it;                // step
  int last;              // the step that leaves w
  uint32_t need;         // the matrix' finished tiles that it waits for
  float* w;
  __nv_bfloat16* out;
};

struct Shared {
  uint64_t full[kStages], empty[kStages];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t in[kBuffers], out[kBuffers], vacant[kBuffers];
  uint64_t listed[kRing], read[kRing], vec[kRing];
  Listed ring[kRing];
  uint32_t tmem;
  volatile int gave_up;
};

// Bounded wait on shared barriers.
__device__ __forceinline__ bool wait_on(Shared& sh, const MuonParams& p,
                                        uint64_t* bar, uint32_t parity) {
  return bounded_wait(bar, parity, &sh.gave_up, p.status,
                      LAMB_STATUS_WAIT_TIMEOUT);
}

// The 16-byte unit q of row r: rows of 64 bytes, rows of 128 bytes.
__device__ __forceinline__ uint32_t unit64(uint32_t base, int r, int q) {
  return base + r * 64 + ((q ^ ((r >> 1) & 3)) << 4);
}
__device__ __forceinline__ uint32_t unit128(uint32_t base, int r, int q) {
  return base + r * 128 + ((q ^ (r & 7)) << 4);
}
// Entry (j, i) of a mirrored block: 32 rows in two halves of 64 columns.
__device__ __forceinline__ uint32_t mirrored(uint32_t base, int j, int i) {
  return unit128(base + (i >> 6) * (kBlockBytes / 2), j, (i & 63) >> 3) +
         (i & 7) * 2;
}
// Whether the block of rows c0 .. and columns a0 .. lies in no tile on or above
// the diagonal.
template <int kCtas>
__device__ __forceinline__ bool mirror(int a0, int c0) {
  return a0 / kTile<kCtas> < c0 / kTile<kCtas>;
}

__device__ __forceinline__ bool ready(const MuonParams& p, const Listed& d) {
  return ld_acquire_u32(p.done + d.matrix) >= d.need;
}
__device__ __forceinline__ bool wait_ready(Shared& sh, const MuonParams& p,
                                           const Listed& d) {
  if (ready(p, d)) return true;
  const uint64_t begin = global_ns();
  while (!ready(p, d)) {
    if (sh.gave_up) return false;
    if (global_ns() - begin > kWaitLimitNs) {
      sh.gave_up = 1;
      atomicOr(p.status, LAMB_STATUS_WAIT_TIMEOUT);
      return false;
    }
    __nanosleep(32);
  }
  return true;
}

// The next listed tile: NULL at the end, or if a wait gave up.
__device__ __forceinline__ const Listed* next_tile(Shared& sh,
                                                   const MuonParams& p,
                                                   int tile) {
  const int slot = tile % kRing;
  if (!wait_on(sh, p, &sh.listed[slot], (uint32_t)(tile / kRing) & 1u))
    return nullptr;
  return sh.ring[slot].phase == kNoTile ? nullptr : &sh.ring[slot];
}

// ---- warp 0 -------------------------------------------------------------------
// Walks over this CTA's or pair's tiles of the list, step after step.
struct Lister {
  int t, units;
  __device__ __forceinline__ void next(const MuonParams& p, Listed& d) {
    d.phase = kNoTile;
    if (t < p.total) {
      const int it = t / p.step_tiles;
      static_cast<MuonTile&>(d) = p.tiles[t - it * p.step_tiles];
      d.it = it;
    }
    t += units;
  }
};

template <int kCtas>
__device__ __forceinline__ void copy_operands(Shared& sh, const MuonParams& p,
                                              uint32_t smem, uint32_t rank) {
  Lister list = {(int)blockIdx.x / kCtas, (int)gridDim.x / kCtas};
  Listed ahead;
  list.next(p, ahead);
  int it = 0;
  for (int n = 0;; ++n) {
    const int slot = n % kRing;
    if (!wait_on(sh, p, &sh.read[slot], ((uint32_t)(n / kRing) & 1u) ^ 1u))
      break;
    Listed& d = sh.ring[slot];
    ahead.last = ahead.phase == kApply && ahead.it == p.steps - 1;
    ahead.need = (uint32_t)(ahead.it * (2 * ahead.sym + ahead.app) +
                            ahead.phase * ahead.sym);
    if (ahead.phase != kNoTile && ahead.last) {
      ahead.w = p.ptrs[ahead.matrix].w;
      ahead.out = p.ptrs[ahead.matrix].out;
    }
    d = ahead;
    mbar_arrive(&sh.listed[slot]);
    if (ahead.phase == kNoTile) break;
    list.next(p, ahead);
    const MuonMatrix* const x = d.x;
    const int from = d.it & 1, kn = d.kn;
    const bool gram_mn = d.phase == kGram && d.tall;
    const bool b_mn = gram_mn || (d.phase == kApply && !d.tall);
    const CUtensorMap *ma, *mb;
    if (d.phase == kGram) {
      ma = mb = d.tall ? &x->x_mn[from] : &x->x_k[from];
    } else if (d.phase == kSquare) {
      ma = mb = &x->d;
    } else {
      ma = d.tall ? &x->x_k[from] : &x->e;
      mb = d.tall ? &x->e : &x->x_mn[from];
    }
    const int a0 = d.i * kTile<kCtas> + (int)rank * kTileM;
    const int b0 = d.j * kTile<kCtas> + (int)rank * kTileM;
    if (!wait_ready(sh, p, d)) break;
    fence_proxy_async();       // other CTAs' blocks, to be read by copies
    for (int kb = 0; kb < kn; ++kb, ++it) {
      const int s = it % kStages;
      if (!wait_on(sh, p, &sh.empty[s], ((uint32_t)(it / kStages) & 1u) ^ 1u))
        break;
      const uint32_t at = smem + s * kStageBytes;
      const int k = kb * kTileK;
      if (rank == 0) mbar_expect(&sh.full[s], kCtas * kStageBytes);
      // (issuing a copy takes this thread some 100 cycles: one an operand)
      if (kCtas == 2) {
        const uint32_t bar = at_rank(&sh.full[s], 0);    // the issuing CTA's
        if (gram_mn) pair_blocks_load(at, ma, k, a0 / 64, bar);
        else pair_tile_load(at, ma, k, a0, bar);
        if (b_mn) pair_blocks_load(at + kTileBytesA, mb, k, b0 / 64, bar);
        else pair_tile_load(at + kTileBytesA, mb, k, b0, bar);
      } else {
        if (gram_mn) blocks_load(at, ma, k, a0 / 64, &sh.full[s]);
        else tile_load(at, ma, k, a0, &sh.full[s]);
        if (b_mn) blocks_load(at + kTileBytesA, mb, k, b0 / 64, &sh.full[s]);
        else tile_load(at + kTileBytesA, mb, k, b0, &sh.full[s]);
      }
    }
    if (sh.gave_up) break;
  }
  // the copies have landed, and the products' arrivals for them are in, before
  // either CTA may leave (cluster_sync)
  for (int j = it > kStages ? it - kStages : 0; j < it; ++j) {
    if (rank == 0 && sh.gave_up)
      settle(&sh.full[j % kStages], (uint32_t)(j / kStages) & 1u);
    wait_on(sh, p, &sh.empty[j % kStages], (uint32_t)(j / kStages) & 1u);
  }
}

// ---- warp 1 -------------------------------------------------------------------
template <int kCtas>
__device__ __forceinline__ void multiply(Shared& sh, const MuonParams& p,
                                         uint32_t smem, uint32_t tmem,
                                         uint32_t rank) {
  int it = 0;
  for (int n = 0; const Listed* d = next_tile(sh, p, n); ++n) {
    const bool a_mn = d->phase == kGram && d->tall;
    const bool b_mn = a_mn || (d->phase == kApply && !d->tall);
    const int kn = d->kn;
    mbar_arrive(&sh.read[n % kRing]);
    if (rank) continue;        // the other CTA issues
    const uint64_t da = operand_desc(a_mn), db = operand_desc(b_mn);
    const uint32_t sa = operand_step(a_mn), sb = operand_step(b_mn);
    const uint32_t desc =
        product_desc(false, a_mn, b_mn, kTile<kCtas>, kTile<kCtas>);
    const int acc = n & 1;
    const uint32_t to = tmem + acc * kTile<kCtas>;
    const uint32_t ph = ((uint32_t)(n >> 1) & 1u) ^ 1u;
    if (!wait_on(sh, p, &sh.acc_empty[acc], ph)) return;
    if (kCtas == 2)
      mbar_try_cluster(&sh.acc_empty[acc], ph);      // the other CTA's readers
    tmem_after_sync();
    for (int kb = 0; kb < kn; ++kb, ++it) {
      const int s = it % kStages;
      if (!wait_on(sh, p, &sh.full[s], (uint32_t)(it / kStages) & 1u)) return;
      tmem_after_sync();
      const uint32_t at = smem + s * kStageBytes;
      const uint64_t a = da | (at >> 4), b = db | ((at + kTileBytesA) >> 4);
#pragma unroll
      for (int k = 0; k < kTileK / 16; ++k) {
        if (kCtas == 2)
          pair_product(to, a + k * sa, b + k * sb, desc, kb > 0 || k > 0);
        else
          product(to, a + k * sa, b + k * sb, desc, kb > 0 || k > 0);
      }
      if (kCtas == 2) pair_products_arrive(&sh.empty[s]);
      else products_arrive(&sh.empty[s]);
    }
    if (kCtas == 2) pair_products_arrive(&sh.acc_full[acc]);
    else products_arrive(&sh.acc_full[acc]);
  }
}

// ---- warp 2 -------------------------------------------------------------------
// This CTA's first row of a tile.
template <int kCtas>
__device__ __forceinline__ int row0(const Listed& d) {
  return d.i * kTile<kCtas> + (kCtas == 2 ? (int)cluster_rank() * kTileM : 0);
}
// Blocks of this CTA's part of a tile: none where that is past the last row.
template <int kCtas>
__device__ __forceinline__ int block_count(const Listed& d) {
  if (row0<kCtas>(d) >= d.height) return 0;
  constexpr int kMost = kTile<kCtas> / kMuonCols;
  const int left =
      (d.width - d.j * kTile<kCtas> + kMuonCols - 1) / kMuonCols;
  return left < kMost ? left : kMost;
}

template <int kCtas>
__device__ __forceinline__ void copy_in(Shared& sh, const MuonParams& p,
                                        uint32_t staging) {
  int n = 0, begun = 0;       // blocks, tiles whose copies were started
  for (int tile = 0; const Listed* l = next_tile(sh, p, tile); ++tile) {
    const Listed& d = *l;
    const MuonMatrix* const x = d.x;
    const int blocks = block_count<kCtas>(d), phase = d.phase;
    const int a0 = row0<kCtas>(d), b0 = d.j * kTile<kCtas>;
    const uint32_t vec = staging + kBuffers * kBufferBytes +
                         tile % kRing * kVecBytes;
    uint64_t* const vb = &sh.vec[tile % kRing];
    const CUtensorMap* const m0 = phase == kSquare ? &x->d_c
                                                   : &x->x_c[d.it & 1];
    if (phase == kGram) {
      mbar_arrive(vb);
    } else {
      if (!wait_ready(sh, p, d)) break;
      fence_proxy_async();
      // the tile's l or beta (their memory goes up to a whole tile)
      const bool cols = phase == kSquare || d.tall;
      const bool rows = phase == kSquare || !d.tall;
      mbar_expect(vb, (cols ? kTile<kCtas> * 4 : 0) + (rows ? kTileM * 4 : 0));
      const float* const v = phase == kSquare ? d.diag : d.beta;
      if (cols) bulk_load_at(vec, v + b0, kTile<kCtas> * 4, vb);
      if (rows) bulk_load_at(vec + kColBytes, v + a0, kTileM * 4, vb);
    }
    begun = tile + 1;
    mbar_arrive(&sh.read[tile % kRing]);
    for (int c = 0; c < blocks; ++c, ++n) {
      const int b = n % kBuffers;
      if (!wait_on(sh, p, &sh.vacant[b], ((uint32_t)(n / kBuffers) & 1u) ^ 1u))
        break;
      const uint32_t to = staging + b * kBufferBytes;
      const int c0 = b0 + c * kMuonCols;
      if (phase == kGram) {
        mbar_arrive(&sh.in[b]);
      } else {
        mbar_expect(&sh.in[b], (phase == kSquare ? 1 : 2) * kBlockBytes);
        tile_load(to, m0, c0, a0, &sh.in[b]);
        if (phase == kApply)
          tile_load(to + kBlockBytes, &x->lo_c, c0, a0, &sh.in[b]);
      }
    }
    if (sh.gave_up) break;
  }
  // copies that were started land before the CTA may leave
  for (int j = n > kBuffers ? n - kBuffers : 0; j < n; ++j)
    settle(&sh.in[j % kBuffers], (uint32_t)(j / kBuffers) & 1u);
  if (begun) settle(&sh.vec[(begun - 1) % kRing],
                    (uint32_t)((begun - 1) / kRing) & 1u);
}

// ---- warp 3 -------------------------------------------------------------------
template <int kCtas>
__device__ __forceinline__ void copy_out(Shared& sh, const MuonParams& p,
                                         uint32_t staging) {
  int n = 0;
  for (int tile = 0; const Listed* l = next_tile(sh, p, tile); ++tile) {
    const MuonMatrix* const x = l->x;
    const int blocks = block_count<kCtas>(*l), m = l->height, matrix = l->matrix;
    const int a0 = row0<kCtas>(*l), b0 = l->j * kTile<kCtas>;
    const int phase = l->phase;
    const bool last = l->last;
    const CUtensorMap* const to = phase == kApply ? &x->x_c[(l->it & 1) ^ 1]
                                  : phase == kGram ? &x->d_c
                                                   : &x->e_c;
    const CUtensorMap* const to_t = phase == kGram ? &x->d_t : &x->e_t;
    mbar_arrive(&sh.read[tile % kRing]);
    for (int c = 0; c < blocks; ++c, ++n) {
      const int b = n % kBuffers;
      if (!wait_on(sh, p, &sh.out[b], (uint32_t)(n / kBuffers) & 1u)) break;
      if (last) {
        mbar_arrive(&sh.vacant[b]);
        continue;
      }
      const uint32_t from = staging + b * kBufferBytes;
      const int c0 = b0 + c * kMuonCols;
      tile_store(to, c0, a0, from);
      if (phase == kApply) {
        tile_store(&x->lo_c, c0, a0, from + kBlockBytes);
      } else if (mirror<kCtas>(a0, c0)) {
        tile_store(to_t, a0, c0, from + kBlockBytes);
        if (a0 + 64 < m)
          tile_store(to_t, a0 + 64, c0,
                     from + kBlockBytes + kBlockBytes / 2);
      }
      stores_commit();
      if (c > 0) {      // the tile's block before
        stores_have_read<1>();
        mbar_arrive(&sh.vacant[(n - 1) % kBuffers]);
      }
    }
    if (!last && blocks) {     // (no blocks: nothing to wait for or to count)
      stores_have_read<0>();
      mbar_arrive(&sh.vacant[(n - 1) % kBuffers]);
      stores_done();
      if (sh.gave_up) break;
      fence_proxy_async();
      __threadfence();
      atomicAdd(p.done + matrix, 1u);
    }
  }
  stores_done();
}

// ---- warps 4-11 -----------------------------------------------------------------
__device__ __forceinline__ void group_sync(int group) {
  asm volatile("bar.sync %0, %1;" ::"r"(kEpiBarrier + group), "n"(kEpiThreads)
               : "memory");
}
// One answer for all of a group.
__device__ __forceinline__ bool group_all(int group, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.pred q, %2, %3, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"((uint32_t)x), "r"(kEpiBarrier + group), "n"(kEpiThreads)
      : "memory");
  return r != 0;
}
// What this thread wrote to staging memory is read by copies from here on.
__device__ __forceinline__ void fence_staging() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ float4 lds_f4(uint32_t at) {
  const uint4 v = lds16(at);
  return make_float4(__uint_as_float(v.x), __uint_as_float(v.y),
                     __uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ float lds_f(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
  return v;
}

struct Row {
  int row, i;            // in the tile, in the matrix
  int group;
  uint32_t col;          // l or beta of the block's columns
  uint32_t buf;
};

// A block of G (kSq: of b G + c G G) without its diagonal, which goes to diag
// (beta); li: the row's l.
template <bool kSq>
__device__ __forceinline__ void symmetric_block(float pb, float pc, int m,
                                                float* diag, float li, float s,
                                                bool both, int c0, const Row& r,
                                                float (&y)[32]) {
  const bool on = r.i >= c0 && r.i < c0 + 32;      // the diagonal
  if (on && r.i < m) {
#pragma unroll
    for (int q = 0; q < 32; ++q)
      if (c0 + q == r.i)
        diag[r.i] = kSq ? pb * li + pc * (li * li + y[q] * s) : y[q] * s;
  }
  if (!kSq) {
#pragma unroll
    for (int q = 0; q < 32; ++q) y[q] *= s * kScaleD;
  } else {
    const float ck = pc * (kScaleE / kScaleD), sk = pc * s * kScaleE;
    const float bk = fmaf(pc, li, pb) * (kScaleE / kScaleD);
    uint4 ds[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) ds[u] = lds16(unit64(r.buf, r.row, u));
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float4 l0 = lds_f4(r.col + 32 * u), l1 = lds_f4(r.col + 32 * u + 16);
      const float l[8] = {l0.x, l0.y, l0.z, l0.w, l1.x, l1.y, l1.z, l1.w};
      const uint4 d = ds[u];
      const uint32_t dw[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int q = 8 * u + k;
        const float2 d2 = half2_at(dw[k >> 1]);
        const float dd = k & 1 ? d2.y : d2.x;
        // E kScaleE, dd being D kScaleD
        y[q] = fmaf(fmaf(ck, l[k], bk), dd, y[q] * sk);
      }
    }
  }
  if (on) {
#pragma unroll
    for (int q = 0; q < 32; ++q)
      if (c0 + q == r.i) y[q] = 0.f;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[k] = pack_half2(y[8 * u + 2 * k], y[8 * u + 2 * k + 1]);
    sts16(unit64(r.buf, r.row, u), make_uint4(w[0], w[1], w[2], w[3]));
    if (both) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        sts2(mirrored(r.buf + kBlockBytes, 8 * u + k, r.row),
             half_bits(w[k >> 1], k & 1));
    }
  }
}

// X <- (a + beta) X + E X of a block; y holds the product and gets X * scale.
template <bool kLast>
__device__ __forceinline__ void apply_block(bool tall, float pa, float br,
                                            const Row& r, float (&y)[32]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    float f[8];
    if (tall) {
      const float4 b0 = lds_f4(r.col + 32 * u), b1 = lds_f4(r.col + 32 * u + 16);
      f[0] = pa + b0.x; f[1] = pa + b0.y; f[2] = pa + b0.z; f[3] = pa + b0.w;
      f[4] = pa + b1.x; f[5] = pa + b1.y; f[6] = pa + b1.z; f[7] = pa + b1.w;
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = br;
    }
    const uint32_t ah = unit64(r.buf, r.row, u), al = ah + kBlockBytes;
    const uint4 hi = lds16(ah), lo = lds16(al);
    const uint32_t hw[4] = {hi.x, hi.y, hi.z, hi.w};
    const uint32_t lw[4] = {lo.x, lo.y, lo.z, lo.w};
    uint32_t oh[4], ol[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 a = half2_at(hw[k]), b = half2_at(lw[k]);
      const int q = 8 * u + 2 * k;
      y[q] = fmaf(f[2 * k], fmaf(b.x, 1.f / kScaleLo, a.x),
                  y[q] * (1.f / kScaleE));
      y[q + 1] = fmaf(f[2 * k + 1], fmaf(b.y, 1.f / kScaleLo, a.y),
                      y[q + 1] * (1.f / kScaleE));
      if (!kLast) {
        oh[k] = pack_half2(y[q], y[q + 1]);
        const float2 h = half2_at(oh[k]);
        ol[k] = pack_half2((y[q] - h.x) * kScaleLo, (y[q + 1] - h.y) * kScaleLo);
      }
    }
    if (!kLast) {
      sts16(ah, make_uint4(oh[0], oh[1], oh[2], oh[3]));
      sts16(al, make_uint4(ol[0], ol[1], ol[2], ol[3]));
    }
  }
}

// The last X to the weights or the direction: eight threads a row of a block.
// The old weights are on their way while the block is turned over.
struct Output {
  float* w;
  __nv_bfloat16* out;
  float inv, keep, move;
  int rows, cols;
  bool step, vec;
};

__device__ __forceinline__ Output output_of(const MuonParams& p,
                                            const Listed& d, float lr) {
  Output o;
  o.w = d.w;
  o.out = d.out;
  o.step = p.d_lr != nullptr;
  o.inv = 1.f / d.scale;
  o.keep = 1.f - lr * p.k.wd * d.decay;
  o.move = lr * muon_size(p.k, d.rows, d.cols);
  o.rows = d.height;
  o.cols = d.width;
  o.vec = d.width % 4 == 0 && (!o.step || (uintptr_t)d.w % 16 == 0) &&
          (uintptr_t)d.out % 8 == 0;
  return o;
}

__device__ __forceinline__ void last_block(const Output& o, int a0, int c0,
                                           const Row& r, float (&y)[32]) {
  const int u = r.row & 7, c = c0 + 4 * u;
  const int cols = min(4, o.cols - c);
  constexpr int kRows = kEpiThreads / 8, kAll = kTileM / kRows;
  float4 old[kAll];
  auto load_old = [&](int k) {
    const int rr = a0 + k * kRows + (r.row >> 3);
    if (o.step && o.vec && cols == 4 && rr < o.rows)
      old[k] = *reinterpret_cast<const float4*>(o.w + (int64_t)rr * o.cols + c);
  };
#pragma unroll
  for (int k = 0; k < kAll / 2; ++k) load_old(k);
  group_sync(r.group);          // everybody has read the block's inputs
#pragma unroll
  for (int q = 0; q < 8; ++q)
    sts16(unit128(r.buf, r.row, q),
          make_uint4(__float_as_uint(y[4 * q] * o.inv),
                     __float_as_uint(y[4 * q + 1] * o.inv),
                     __float_as_uint(y[4 * q + 2] * o.inv),
                     __float_as_uint(y[4 * q + 3] * o.inv)));
#pragma unroll
  for (int k = kAll / 2; k < kAll; ++k) load_old(k);     // (y is gone)
  group_sync(r.group);
#pragma unroll
  for (int k = 0; k < kAll; ++k) {
    const int br = k * kRows + (r.row >> 3), rr = a0 + br;
    const uint4 b = lds16(unit128(r.buf, br, u));
    if (rr >= o.rows || cols <= 0) continue;
    float v[4] = {__uint_as_float(b.x), __uint_as_float(b.y),
                  __uint_as_float(b.z), __uint_as_float(b.w)};
    const int64_t at = (int64_t)rr * o.cols + c;
    if (o.vec && cols == 4) {
      if (o.step) {
        v[0] = o.keep * old[k].x - o.move * v[0];
        v[1] = o.keep * old[k].y - o.move * v[1];
        v[2] = o.keep * old[k].z - o.move * v[2];
        v[3] = o.keep * old[k].w - o.move * v[3];
        *reinterpret_cast<float4*>(o.w + at) =
            make_float4(v[0], v[1], v[2], v[3]);
      }
      if (o.out) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[0], v[1]);
        const __nv_bfloat162 l = __floats2bfloat162_rn(v[2], v[3]);
        *reinterpret_cast<uint2*>(o.out + at) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&h),
                       *reinterpret_cast<const uint32_t*>(&l));
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q >= cols) break;
        if (o.step) {
          v[q] = o.keep * o.w[at + q] - o.move * v[q];
          o.w[at + q] = v[q];
        }
        if (o.out) o.out[at + q] = __float2bfloat16_rn(v[q]);
      }
    }
  }
}

template <int kCtas>
__device__ __forceinline__ void turn_over(Shared& sh, const MuonParams& p,
                                          uint32_t staging, uint32_t tmem) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int quarter = warp & 3;
  Row r;
  r.row = quarter * 32 + lane;
  r.group = (warp - 4) >> 2;
  const float lr = p.d_lr ? *p.d_lr : 0.f;
  const float pa = p.k.a, pb = p.k.b, pc = p.k.c;
  int n = 0;
  for (int tile = 0;; ++tile) {
    const int slot = tile % kRing, acc = tile & 1;
    // one answer for all: the last step's blocks meet at barriers
    bool ok = wait_on(sh, p, &sh.listed[slot], (uint32_t)(tile / kRing) & 1u);
    if (!group_all(r.group, ok)) return;
    const Listed* const l = &sh.ring[slot];
    if (l->phase == kNoTile) return;
    ok = wait_on(sh, p, &sh.acc_full[acc], (uint32_t)(tile >> 1) & 1u);
    if (!group_all(r.group, ok)) return;
    tmem_after_sync();
    const uint32_t from =
        tmem + acc * kTile<kCtas> + ((uint32_t)(quarter * 32) << 16);
    const int a0 = row0<kCtas>(*l), b0 = l->j * kTile<kCtas>;
    const int blocks = block_count<kCtas>(*l), phase = l->phase, m = l->height;
    const bool last = l->last, tall = l->tall;
    r.i = a0 + r.row;
    const float s = phase == kGram ? 1.f / (l->scale * l->scale)
                                   : 1.f / (kScaleD * kScaleD);
    float* const diag = phase == kGram ? l->diag : l->beta;
    const uint32_t vec = staging + kBuffers * kBufferBytes + slot * kVecBytes;
    float row_v = 0.f;            // the row's l or beta
    Output o;
    if (last) o = output_of(p, *l, lr);
    if (phase != kGram) {
      wait_on(sh, p, &sh.vec[slot], (uint32_t)(tile / kRing) & 1u);
      row_v = lds_f(vec + kColBytes + 4 * r.row);
    }
    for (int c = 0; c < blocks; ++c, ++n) {
      if (n % kGroups != r.group) continue;
      const int b = n % kBuffers, c0 = b0 + c * kMuonCols;
      r.buf = staging + b * kBufferBytes;
      r.col = vec + c * (kMuonCols * 4);
      float y[32];
      tmem_ld32(from + c * kMuonCols, y);
      wait_on(sh, p, &sh.in[b], (uint32_t)(n / kBuffers) & 1u);
      if (phase == kGram) {
        symmetric_block<false>(pb, pc, m, diag, 0.f, s, mirror<kCtas>(a0, c0),
                               c0, r, y);
      } else if (phase == kSquare) {
        symmetric_block<true>(pb, pc, m, diag, row_v, s, mirror<kCtas>(a0, c0),
                              c0, r, y);
      } else if (!last) {
        apply_block<false>(tall, pa, pa + row_v, r, y);
      } else {
        apply_block<true>(tall, pa, pa + row_v, r, y);
        last_block(o, a0, c0, r, y);
      }
      fence_staging();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.out[b]);
    }
    tmem_before_sync();
    __syncwarp();
    if (lane == 0) {
      if (kCtas == 2) remote_arrive(at_rank(&sh.acc_empty[acc], 0));
      else mbar_arrive(&sh.acc_empty[acc]);
      mbar_arrive(&sh.read[slot]);
    }
  }
}

template <int kCtas>
__global__ void __cluster_dims__(kCtas, 1, 1)
    __launch_bounds__(kStepThreads, 1)
muon_steps_kernel(const __grid_constant__ MuonParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ Shared sh;
  const int warp = threadIdx.x >> 5;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t staging = smem + kStages * kStageBytes;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.acc_full[i], 1);
      mbar_init(&sh.acc_empty[i], 4 * kGroups * kCtas);
    }
    for (int i = 0; i < kBuffers; ++i) {
      mbar_init(&sh.in[i], 1);
      mbar_init(&sh.out[i], kEpiThreads / 32);
      mbar_init(&sh.vacant[i], 1);
    }
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&sh.listed[i], 1);
      mbar_init(&sh.read[i], kReaders);
      mbar_init(&sh.vec[i], 1);
    }
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  if (warp == 2) {
    if (kCtas == 2) pair_tmem_alloc_all(&sh.tmem);
    else tmem_alloc_all(&sh.tmem);
  }
  for (int i = threadIdx.x; i < p.n_mats * kMuonMaps; i += kStepThreads)
    take_map(reinterpret_cast<const CUtensorMap*>(p.mats + i / kMuonMaps) +
             i % kMuonMaps);
  tmem_before_sync();
  __syncthreads();
  if (kCtas == 2) cluster_sync();        // both CTAs' barriers are there
  tmem_after_sync();
  const uint32_t tmem = sh.tmem, rank = kCtas == 2 ? cluster_rank() : 0;
  if (warp == 0) {
    if (elect_lane()) copy_operands<kCtas>(sh, p, smem, rank);
    __syncwarp();
  } else if (warp == 1) {
    if (elect_lane()) multiply<kCtas>(sh, p, smem, tmem, rank);
    __syncwarp();
  } else if (warp == 2) {
    if (elect_lane()) copy_in<kCtas>(sh, p, staging);
    __syncwarp();
  } else if (warp == 3) {
    if (elect_lane()) copy_out<kCtas>(sh, p, staging);
    __syncwarp();
  } else {
    turn_over<kCtas>(sh, p, staging, tmem);
  }
  tmem_before_sync();
  __syncthreads();
  if (kCtas == 2) cluster_sync();        // neither's memory is used any more
  tmem_after_sync();
  if (warp == 2) {
    if (kCtas == 2) pair_tmem_free_all(tmem);
    else tmem_free_all(tmem);
  }
}

}  // namespace

template <int kCtas>
cudaError_t muon_setup(int sms, int* units) {
  cudaError_t e = cudaFuncSetAttribute(
      muon_steps_kernel<kCtas>, cudaFuncAttributeMaxDynamicSharedMemorySize,
      (int)kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = kCtas;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(sms / kCtas * kCtas));
  cfg.blockDim = dim3(kStepThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(units, muon_steps_kernel<kCtas>, &cfg);
  if (e == cudaSuccess && *units < 1) e = cudaErrorNotSupported;
  return e;
}

cudaError_t muon_steps_setup(int sms, int* ctas, int* pairs) {
  const cudaError_t e = muon_setup<1>(sms, ctas);
  return e == cudaSuccess ? muon_setup<2>(sms, pairs) : e;
}

cudaError_t muon_launch_steps(const MuonParams& p, bool pair, int units,
                              cudaStream_t stream) {
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeCooperative;
  at.val.cooperative = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kStepThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  // a process that has fewer SMs than the device takes fewer CTAs
  cudaError_t e = cudaErrorCooperativeLaunchTooLarge;
  for (int n = std::min(units, p.total);
       n > 0 && e == cudaErrorCooperativeLaunchTooLarge; n /= 2) {
    cfg.gridDim = dim3((unsigned)(pair ? 2 * n : n));
    e = cudaLaunchKernelEx(
        &cfg, pair ? muon_steps_kernel<2> : muon_steps_kernel<1>, p);
    if (e == cudaErrorCooperativeLaunchTooLarge) cudaGetLastError();
  }
  return e;
}

}  // namespace lamb
