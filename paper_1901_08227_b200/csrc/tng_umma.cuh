// Tensor-memory matrix instructions on 8-bit integers, tiled copies and cluster barriers (sm_100a).
//
// Operand tiles are rows of 128 bytes (128 codes of the contraction), copied by TMA with the 128-byte
// swizzle: groups of eight rows make 1024-byte atoms, one after the other.  The matrix descriptor names the
// atom pitch and the swizzle; a step of 32 codes along the contraction moves its start address by 32 bytes.
#pragma once

#include <cuda.h>

#include "tng_pipeline.cuh"

namespace tng {

// ---- descriptors ---------------------------------------------------------------------------------
// Shared-memory matrix descriptor of a K-major tile in the 128-byte swizzle, at a 1024-byte aligned
// address: start >> 4 (bits 0-13), leading offset (unused with this layout, 1), stride between eight-row
// atoms 1024 >> 4 (bits 32-45), version 1 (bits 46-47), swizzle code 2 (bits 61-63).
__device__ __forceinline__ uint64_t umma_desc(uint32_t smem) {
    return ((uint64_t)(smem & 0x3FFFFu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor, kind::i8: int32 accumulator (2 at bit 4), signed 8-bit A and B (1 at bits 7 and
// 10), both K-major, N >> 3 at bit 17, M >> 4 at bit 24.
__host__ __device__ constexpr uint32_t umma_idesc_s8(uint32_t m, uint32_t n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | ((m >> 4) << 24);
}

// One instruction: D (+)= A B^T over 32 codes, issued by one thread (of the even CTA with GROUP = 2).
template <int GROUP>
__device__ __forceinline__ void umma_s8(uint32_t tmem, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    if constexpr (GROUP == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem), "l"(a), "l"(b), "r"(idesc),
                     "r"((uint32_t)accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem), "l"(a), "l"(b), "r"(idesc),
                     "r"((uint32_t)accumulate) : "memory");
}
// Arrive on a barrier when every instruction issued so far is done: this CTA's, or the same one of the CTAs of a mask.
__device__ __forceinline__ void umma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void umma_commit_pair(uint32_t bar, uint16_t ctas) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(ctas) : "memory");
}
__device__ __forceinline__ void umma_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void umma_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// ---- tensor memory -------------------------------------------------------------------------------
// Whole warp; with GROUP = 2 one warp of each CTA of the pair.  The address lands in shared memory.
template <int GROUP> __device__ __forceinline__ void tmem_alloc(uint32_t dst_smem, uint32_t columns) {
    if constexpr (GROUP == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int GROUP> __device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns) {
    if constexpr (GROUP == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
// 32 (16) columns of the warp's 32 lanes; lane i of the warp gets row i.  Complete when tmem_wait_ld returns.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- tiled copies --------------------------------------------------------------------------------
// A box of the map at (x = first code, y = first row) into this CTA's shared memory; completion on `bar`, a
// shared::cluster address (GROUP = 2: may be the pair's even CTA's).  x is a multiple of 128 here, so the
// copy starts on a 16-byte boundary.
template <int GROUP> __device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
    if constexpr (GROUP == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// This CTA's shared memory into a box of the map, clipped to the matrix, whose rows are whole 16-byte pieces; x a multiple of
// 16 bytes, both >= 0.
__device__ __forceinline__ void tile_store(const CUtensorMap* map, int32_t x, int32_t y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// Until at most N of this thread's stores still read shared memory.
template <int N> __device__ __forceinline__ void tile_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void tile_store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// This thread's shared-memory writes become visible to copies issued after the next barrier.
__device__ __forceinline__ void smem_to_copies() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void map_prefetch(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ---- clusters ------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Its two halves: the release orders this thread's accesses, reads of other CTAs' memories among them, before the
// arrival, so that past the wait nobody's are under way.  (Stores to global memory between the halves are not waited for.)
__device__ __forceinline__ void cluster_arrive_all() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait_all() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// A mere meeting point: nothing is made visible or waited for (no wait for stores).
__device__ __forceinline__ void cluster_meet_all() {
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// Address of `smem` (this CTA's) in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t cluster_map(uint32_t smem, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem), "r"(rank));
    return r;
}
// Relaxed: it orders nothing but what tensor-memory fences order (a release here waits 1500 cycles for stores).
__device__ __forceinline__ void cluster_arrive(uint32_t remote_bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote_bar) : "memory");
}
__device__ __forceinline__ int cluster_ld(uint32_t remote) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(remote) : "memory");
    return v;
}

__device__ __forceinline__ int4 cluster_ld4(uint32_t remote) {              // 16-byte aligned
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(remote) : "memory");
    return v;
}
// Whether a flag word of every CTA of the cluster is zero (whole warp, n <= 32 CTAs).
__device__ __forceinline__ bool cluster_all_zero(uint32_t flag, uint32_t n) {
    const uint32_t lane = threadIdx.x & 31;
    return __all_sync(0xFFFFFFFFu, lane >= n || cluster_ld(cluster_map(flag, lane)) == 0);
}

}  // namespace tng
