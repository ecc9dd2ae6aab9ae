// Building blocks for tcgen05 on pairs of CTAs, beside those of umma.cuh: operand
// descriptors of any layout, cluster barriers, pair MMAs, 16-byte asynchronous
// copies.  Written from the PTX ISA.
#pragma once

#include "umma.cuh"

namespace hwr {
namespace umma {

// ---- descriptors ---------------------------------------------------------------

// Shared-memory matrix descriptor of any layout: lbo and sbo in bytes, swizzle
// 2, 4 or 6 for 128, 64 or 32 bytes.  K-major: rows of the swizzle's
// width, sbo bytes between groups of 8 rows (lbo unused).  MN-major, 128-byte
// swizzle: 64 16-bit elements of the M (or N) side a row, one row per K index,
// sbo bytes between groups of 8 K indices, lbo between blocks of 64 elements.
__device__ __forceinline__ uint64_t sdesc(uint32_t saddr, uint32_t lbo, uint32_t sbo, uint32_t swizzle) {
    return (uint64_t)((saddr & 0x3FFFF) >> 4) | (uint64_t)((lbo >> 4) & 0x3FFF) << 16 |
           (uint64_t)((sbo >> 4) & 0x3FFF) << 32 | (uint64_t)1 << 46 | (uint64_t)swizzle << 61;
}

// Instruction descriptor, kind::f16, fp32 D: A and B both bf16 or both fp16,
// each K-major or MN-major.
__host__ __device__ constexpr uint32_t idesc_16bit(int M, int N, bool f16, bool a_mn, bool b_mn) {
    return (1u << 4) | (f16 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)a_mn << 15) |
           ((uint32_t)b_mn << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// ---- CTA pairs (clusters of two) ---------------------------------------------
//
// An MMA of cta_group::2 is issued by one thread of the pair's even CTA: D has
// 256 rows, 128 in each CTA's TMEM; each CTA's shared memory holds its 128 rows
// of A and its half of B's N rows, at the same offsets.

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Shared-memory address of `p` in the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t smem_of(const void *p, uint32_t rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}

// Arrive on a barrier of any CTA of the cluster (address from smem_of).  It
// orders execution alone (waited for with mbar_wait<true>), which is all that
// tensor memory needs between the tcgen05 fences of both sides.  Shared memory
// written by threads needs the two fences below too.  (An arrival that releases
// covers global memory and waits a round trip to L2: 64 rows through 12 experts of
// 1,024 x 4,096 took 32 us with it, 27 with the fences.)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}

// Before such an arrival: what this CTA's shared memory holds by then, for those
// who wait.  After the wait: what the cluster's CTAs have released so.
__device__ __forceinline__ void fence_release_smem() {
    asm volatile("fence.release.sync_restrict::shared::cta.cluster;" ::: "memory");
}
__device__ __forceinline__ void fence_acquire_smem() {
    asm volatile("fence.acquire.sync_restrict::shared::cluster.cluster;" ::: "memory");
}

// Tiled 3-D load into this CTA's shared memory that completes its bytes on a
// barrier of either CTA of the pair (address from smem_of).
__device__ __forceinline__ void tma_load_3d_pair(void *dst, const CUtensorMap *map, uint32_t bar,
                                                 int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
        "l"((uint64_t)map), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}

__device__ __forceinline__ void tmem_alloc_pair(uint32_t *dst_smem, uint32_t ncols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(dst_smem)),
                 "r"(ncols)
                 : "memory");
}

__device__ __forceinline__ void tmem_relinquish_pair() {
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
                 : "memory");
}

__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                         uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// As mma_pair, accumulating, and leaving alone the D rows whose bit is set in
// off[row / 32] (rows 128 to 255: the odd CTA's).
__device__ __forceinline__ void mma_pair_rows(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                              uint32_t idesc, const uint32_t (&off)[8]) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%4, %5, %6, %7, %8, %9, %10, %11}, p;\n\t}" ::"r"(
            d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]),
        "r"(off[4]), "r"(off[5]), "r"(off[6]), "r"(off[7])
        : "memory");
}

// Arrive once on `bar` of both CTAs of the pair when all MMAs issued so far finish.
__device__ __forceinline__ void mma_commit_pair(uint64_t *bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
}

// ---- asynchronous copies of 16 bytes -------------------------------------------

// The first `bytes` (0 to 16) bytes from src, then zeros.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// One of the barrier's arrivals, made once all of this thread's cp_async16 so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint64_t *bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

}  // namespace umma
}  // namespace hwr
