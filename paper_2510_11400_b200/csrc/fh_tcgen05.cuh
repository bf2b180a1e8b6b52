// Tensor-core instructions of sm_100a as the product kernels use them: tensor memory, scale copies, matrix instructions on 4-bit
// operands with block scales and on 8-bit integers, clusters.
#pragma once

#include <stdint.h>

#include "fh_device.cuh"

namespace fh {

__device__ __forceinline__ void tmem_alloc(uint32_t* at, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(at)), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_last_alloc() { asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Arrives at `bar` when all matrix instructions and scale copies that this thread has issued are complete.
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Shared-memory descriptor without swizzle: the operand is made of pieces of 8 rows x 16 bytes, each 128 bytes in a row; `lead`
// bytes from a piece to the next along a row, `stride` bytes to the next eight rows.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
  return (uint64_t)(addr >> 4 & 0x3FFFu) | (uint64_t)(lead >> 4 & 0x3FFFu) << 16 | (uint64_t)(stride >> 4 & 0x3FFFu) << 32 | 1ull << 46;
}

// 512 bytes of scales (128 rows, four blocks) to four columns of tensor memory, repeated for each 32 lanes.
__device__ __forceinline__ void tc_copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

// Instruction descriptor: both operands E2M1, M x N, scales E8M0 or E4M3; `id`: which of a word's scales come first.
__host__ __device__ constexpr uint32_t mx_idesc(uint32_t m, uint32_t n, bool e8m0, uint32_t id) {
  return id << 4 | 1u << 7 | 1u << 10 | n / 8u << 17 | (e8m0 ? 1u : 0u) << 23 | m / 16u << 24 | id << 29;
}

// D (+)= A B^T over 64 elements: block-scaled, blocks of 32 (two scales to a row) or 16 (four).
template <bool B32>
__device__ __forceinline__ void tc_mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
  if (B32)
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)add)
        : "memory");
}

// Instruction descriptor: both operands signed 8-bit integers, sums in 32 bits, M x N.
__host__ __device__ constexpr uint32_t i8_idesc(uint32_t m, uint32_t n) { return 2u << 4 | 1u << 7 | 1u << 10 | n / 8u << 17 | m / 16u << 24; }
// D (+)= A B^T over 32 elements; with PAIR of a pair of CTAs (see below).
template <bool PAIR>
__device__ __forceinline__ void tc_mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  if (PAIR)
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}

// ---- a pair of CTAs (neighbouring ranks of a cluster) on one accumulator: 256 rows, 128 in each CTA's tensor memory.  The even one issues;
// an address is that in either CTA's own memory.
__device__ __forceinline__ void tmem_alloc_pair(uint32_t* at, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(at)), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t base, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_last_alloc_pair() { asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory"); }
// Arrives at `bar` of both CTAs.
__device__ __forceinline__ void tc_commit_pair(uint64_t* bar, uint16_t mask) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"(mask)
               : "memory");
}
// Each CTA's scales to its own tensor memory.
__device__ __forceinline__ void tc_copy_scales_pair(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <bool B32>
__device__ __forceinline__ void tc_mma_mx_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
  if (B32)
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)add)
        : "memory");
}
// Takes `bytes` that will not come off what the current phase waits for.
__device__ __forceinline__ void mbar_complete_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// Address of this CTA's `p` in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t at_rank(const void* p, uint32_t rank) {
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(p)), "r"(rank));
  return there;
}
// A box of a tensor map to this CTA's memory, told to a barrier that may be the pair's other CTA's (`bar`: its cluster address).
__device__ __forceinline__ void tma_pair_3d(uint32_t dst, const void* map, uint32_t x, uint32_t y, uint32_t z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_pair_2d(uint32_t dst, const void* map, uint32_t x, uint32_t y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
// Arrival at the same barrier of CTA `rank`, after all that this thread has seen; and the wait that sees it (bounded).
__device__ __forceinline__ void mbar_arrive_at(uint64_t* bar, uint32_t rank) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(at_rank(bar, rank)) : "memory");
}
// Polls without pause: a suspended thread wakes up late, and a stage of these kernels takes less than that (see mx_product_kernel).
// The limit, a kernel argument, is looked at every 16 polls (in each of them: 4096 x 4096 x 4096 43.7 us, with a
// constant 42.5).
// CLUSTER: what is waited for was written by another CTA's thread.
template <bool CLUSTER>
__device__ __forceinline__ bool mbar_poll(uint64_t* bar, uint32_t parity, uint32_t limit, const volatile uint32_t* abort) {
  for (uint32_t i = 0;; ++i) {
    uint32_t ok;
    if (CLUSTER)
      asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                   : "=r"(ok)
                   : "r"(smem_u32(bar)), "r"(parity)
                   : "memory");
    else
      asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                   : "=r"(ok)
                   : "r"(smem_u32(bar)), "r"(parity)
                   : "memory");
    if (ok) return true;
    if ((i & 15u) == 15u && (*abort || i >= limit)) return false;
  }
}

// The same for a whole warp, one lane of which looks.
__device__ __forceinline__ bool mbar_poll_warp(uint64_t* bar, uint32_t parity, uint32_t limit, const volatile uint32_t* abort) {
  bool ok = true;
  if (threadIdx.x % 32 == 0) ok = mbar_poll<true>(bar, parity, limit, abort) && !*abort;
  return __all_sync(0xFFFFFFFFu, ok);
}

// 16 columns of the warp's 32 lanes: lane i gets its row's.  The values are there after tc_load_wait().
__device__ __forceinline__ void tc_load16(uint32_t tmem, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(tmem)
      : "memory");
}
// One column.
__device__ __forceinline__ uint32_t tc_load1(uint32_t tmem) {
  uint32_t v;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(v) : "r"(tmem) : "memory");
  return v;
}
__device__ __forceinline__ void tc_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Sets this CTA's flag in all `ctas` CTAs of the cluster, for whoever is behind the next cluster_sync(), or polls it.
__device__ __forceinline__ void raise_cluster(volatile uint32_t* flag, uint32_t ctas) {
#pragma unroll 1
  for (uint32_t r = 0; r < ctas; ++r) asm volatile("st.volatile.shared::cluster.u32 [%0], %1;" ::"r"(at_rank(const_cast<uint32_t*>(flag), r)), "r"(1u) : "memory");
}
__device__ __forceinline__ uint32_t ld_cluster_u32(const void* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at_rank(p, rank)) : "memory");
  return v;
}
// Word at `addr` of the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ float ld_cluster(uint32_t addr, uint32_t rank) {
  uint32_t there;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there) : "memory");
  return v;
}

}  // namespace fh
