// PTX of the tensor-core products (lm_gemm.cuh): tensor copies, matrix
// descriptors, tcgen05 products with accumulators in tensor memory, and waits
// that give up.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "lamb_sync.cuh"

namespace lamb {
namespace {

// ---- bounded waits ----------------------------------------------------------
// A wait of a product's CTA for its own copies, products or readers ends within
// microseconds.  One that lasts kWaitLimitNs sets the CTA's flag and the status
// word, and every role leaves its loop.
constexpr uint64_t kWaitLimitNs = 2000000000ull;

__device__ __forceinline__ bool bounded_wait(uint64_t* bar, uint32_t parity,
                                             volatile int* gave_up,
                                             uint32_t* status, uint32_t bit) {
  if (mbar_try(bar, parity)) return true;
  const uint64_t begin = global_ns();
  while (!mbar_try(bar, parity)) {
    if (*gave_up) return false;
    if (global_ns() - begin > kWaitLimitNs) {
      *gave_up = 1;
      atomicOr(status, bit);
      return false;
    }
  }
  return true;
}

// Waits, whatever happened, for a copy that was issued.
__device__ __forceinline__ void settle(uint64_t* bar, uint32_t parity) {
  const uint64_t begin = global_ns();
  while (!mbar_try(bar, parity))
    if (global_ns() - begin > kWaitLimitNs) return;
}

// One lane of a converged warp.
__device__ __forceinline__ bool elect_lane() {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok));
  return ok != 0;
}

// Tensor maps that lie in global memory and were written by a copy from the host:
// before a CTA uses one, a thread of it has to take it over (and a barrier to
// follow).  Without it a copy may go by the map that was at the address before.
__device__ __forceinline__ void take_map(const CUtensorMap* map) {
  asm volatile("fence.proxy.tensormap::generic.acquire.sys [%0], 128;"
               ::"l"(map) : "memory");
}

// ---- tensor copies ----------------------------------------------------------
__device__ __forceinline__ void tile_load(uint32_t smem, const CUtensorMap* map,
                                          int x, int y, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile"
      ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(smem), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
      : "memory");
}

// bulk_load to a shared-memory address.
__device__ __forceinline__ void bulk_load_at(uint32_t smem, const void* gmem,
                                             uint32_t bytes, uint64_t* b) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1], %2, [%3];"
      ::"r"(smem), "l"(gmem), "r"(bytes), "r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void blocks_load(uint32_t smem,
                                            const CUtensorMap* map, int line,
                                            int block, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile"
      ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(smem), "l"(map), "r"(0), "r"(line), "r"(block), "r"(smem_u32(bar))
      : "memory");
}
// Shared memory to a tensor; part of the thread's open group of stores.
__device__ __forceinline__ void tile_store(const CUtensorMap* map, int x, int y,
                                           uint32_t smem) {
  asm volatile(
      "cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group "
      "[%0, {%1, %2}], [%3];"
      ::"l"(map), "r"(x), "r"(y), "r"(smem)
      : "memory");
}
// The same, added to what is there (fp32).
__device__ __forceinline__ void tile_add(const CUtensorMap* map, int x, int y,
                                         uint32_t smem) {
  asm volatile(
      "cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group "
      "[%0, {%1, %2}], [%3];"
      ::"l"(map), "r"(x), "r"(y), "r"(smem)
      : "memory");
}
__device__ __forceinline__ void stores_commit() {
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// All but the thread's newest kNewest groups have read shared memory.
template <int kNewest>
__device__ __forceinline__ void stores_have_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kNewest) : "memory");
}
__device__ __forceinline__ void stores_done() {
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}
// Staging memory.  Not "memory": these keep their order among themselves and to
// the barriers, and other loads may move past them.
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ void sts16(uint32_t at, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};"
               ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w));
}
__device__ __forceinline__ void sts2(uint32_t at, uint16_t v) {
  asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(v));
}

// ---- pairs of CTAs ------------------------------------------------------------
// Two CTAs of a cluster multiply one tile of 256 x 256: each holds 128 rows of A
// and of B and gets 128 rows of the accumulator; the even one issues.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile(
      "barrier.cluster.arrive.release.aligned;\n\t"
      "barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same shared variable of CTA `rank`.
__device__ __forceinline__ uint32_t at_rank(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
               : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ void remote_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];"
               ::"r"(bar) : "memory");
}
// mbar_try for arrivals from the other CTA.
__device__ __forceinline__ bool mbar_try_cluster(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
  return ok != 0;
}
// Copies into this CTA's shared memory, counted by a barrier of either CTA.
__device__ __forceinline__ void pair_tile_load(uint32_t smem,
                                               const CUtensorMap* map, int x,
                                               int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile"
      ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(smem), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_blocks_load(uint32_t smem,
                                                 const CUtensorMap* map,
                                                 int line, int block,
                                                 uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile"
      ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(smem), "l"(map), "r"(0), "r"(line), "r"(block), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void pair_product(uint32_t tmem, uint64_t a,
                                             uint64_t b, uint32_t desc,
                                             bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
      : "memory");
}
// Arrives at the barrier's place in both CTAs once the products are complete.
__device__ __forceinline__ void pair_products_arrive(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster"
      ".multicast::cluster.b64 [%0], %1;"
      ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void pair_tmem_alloc_all(uint32_t* smem_out) {
  asm volatile(
      "tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\n\t"
      "tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;"
      :: "r"(smem_u32(smem_out)) : "memory");
}
__device__ __forceinline__ void pair_tmem_free_all(uint32_t base) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;"
               :: "r"(base) : "memory");
}

// ---- products ---------------------------------------------------------------
// Descriptor of a shared-memory operand in the 128-byte swizzle (start address
// added later, all in units of 16 bytes).  K-major: rows of 64 elements (128
// bytes), eight rows to a swizzle pattern of 1024 bytes.  MN-major: blocks of 64
// rows of the operand by 64 of K, a line of 128 bytes for each k; the next 64
// rows are a block (8192 bytes) on, the next eight k 1024 bytes.
__device__ __forceinline__ uint64_t operand_desc(bool mn_major) {
  const uint64_t lbo = mn_major ? 8192 >> 4 : 1;
  const uint64_t sbo = 1024 >> 4;
  return (lbo << 16) | (sbo << 32) | (1ull << 46) | (2ull << 61);
}
// 16 elements further along K.
__device__ __forceinline__ uint32_t operand_step(bool mn_major) {
  return (mn_major ? 16 * 128 : 32) >> 4;
}
// Accumulators in fp32; the operands both bf16 or both fp16.
__device__ __forceinline__ uint32_t product_desc(bool bf16, bool a_mn,
                                                 bool b_mn, int m, int n) {
  const uint32_t f = bf16 ? 1u : 0u;
  return (1u << 4) | (f << 7) | (f << 10) | ((a_mn ? 1u : 0u) << 15) |
         ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void product(uint32_t tmem, uint64_t a, uint64_t b,
                                        uint32_t desc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
      : "memory");
}
// Arrives at the barrier once the products issued so far are complete.
__device__ __forceinline__ void products_arrive(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 "
      "[%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_before_sync() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tmem_after_sync() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// 32 consecutive columns of the warp's 32 lanes: lane i gets its row's values.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&x)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, "
      "%30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
        "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(addr));
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}

}  // namespace
}  // namespace lamb
