// The instructions that feed and run the tensor cores of sm_100a: memory barriers in shared memory, bulk and tiled copies into
// it, tensor memory, and the block-scaled 4-bit multiply.
#pragma once

#include <cuda.h>

#include "uq_device.cuh"

namespace uq {

// ---- barriers -----------------------------------------------------------------------------------

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_init_visible() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

// Waits until the barrier's phase of that parity is complete, for about two seconds at most; false, and *gave_up set for the
// CTA's other waits to see, if it is not by then.  (No timer is read while a wait is short.)
constexpr long long kWaitCycles = 4000000000ll;
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile int *gave_up)
{
    long long start = 0;
    for (uint32_t i = 1;; ++i) {
        if (barrier_try(bar, parity)) return true;
        if ((i & 255u) == 0) {
            const long long now = clock64();
            if (start == 0) start = now;
            if (*gave_up != 0 || now - start > kWaitCycles) break;
        }
    }
    *gave_up = 1;
    return false;
}

// The same by a whole warp, its lanes together.  (The warps that copy and multiply stay together and elect a lane where something is
// issued: 8192^3 200 us against 329 from a branch that one lane takes.)
__device__ __forceinline__ bool barrier_wait_warp(uint32_t bar, uint32_t parity, volatile int *gave_up)
{
    long long start = 0;
    for (uint32_t i = 1;; ++i) {
        if (__all_sync(0xFFFFFFFFu, barrier_try(bar, parity))) return true;
        if ((i & 255u) == 0) {
            const long long now = clock64();
            if (start == 0) start = now;
            if (__any_sync(0xFFFFFFFFu, *gave_up != 0 || now - start > kWaitCycles)) break;
        }
    }
    *gave_up = 1;
    return false;
}

// True in one lane of a converged warp.
__device__ __forceinline__ bool elect_lane()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// ---- clusters -----------------------------------------------------------------------------------

// An arrival at a barrier of any CTA of the cluster.  It orders nothing that this thread has written to memory (a release would
// wait for all its stores): what it says is that tensor memory has been read.
__device__ __forceinline__ void cluster_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ float4 cluster_load4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// ---- copies into shared memory ------------------------------------------------------------------

// bytes: a multiple of 16; both addresses 16-byte aligned.
__device__ __forceinline__ void copy_bulk(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void copy_tile(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// The same for a pair of CTAs: into this CTA's memory, with the barrier (an address in the cluster) in either.
__device__ __forceinline__ void copy_tile_pair(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// ---- tensor memory ------------------------------------------------------------------------------

// CTAS = 2: the two CTAs of a pair work as one.  Allocation and release are by one whole warp (of both CTAs); `columns` a power
// of two from 32 to 512; the address lands in shared memory.
template <int CTAS> __device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t columns)
{
    if constexpr (CTAS == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(dst), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(dst), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int CTAS> __device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns)
{
    if constexpr (CTAS == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(columns));
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 16 columns of the calling warp's 32 lanes, one lane per thread.
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// 512 bytes of scales (32 rows of 16 bytes in shared memory) into four columns, the same in each group of 32 lanes; CTAS = 2: in
// either CTA from its own shared memory.
template <int CTAS> __device__ __forceinline__ void tmem_copy_scales(uint32_t tmem, uint64_t desc)
{
    if constexpr (CTAS == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" :: "r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" :: "r"(tmem), "l"(desc) : "memory");
}

// The barrier (CTAS = 2: that of both CTAs) gets an arrival when everything that this thread has issued to the tensor core is done.
template <int CTAS> __device__ __forceinline__ void tensor_commit(uint32_t bar)
{
    if constexpr (CTAS == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     :: "r"(bar), "h"((uint16_t)3) : "memory");
}

// Shared-memory operand descriptors (address in 16-byte units; bit 46: the sm_100 form).  Matrix rows of 128 bytes in the
// 128-byte swizzle, groups of eight rows 1024 bytes apart; scales without a swizzle, groups of eight 16-byte rows 128 apart.
__device__ __forceinline__ uint64_t operand_descriptor(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ uint64_t scales_descriptor(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

// Instruction descriptor of the block-scaled 4-bit multiply: E2M1 operands (1 at bits 7 and 10), N / 8 at bit 17, E8M0 scales
// (bit 23), M / 128 at bit 27; which half of a column's four scales it uses goes to bits 4 (B) and 29 (A), 0 or 2.
__host__ __device__ constexpr uint32_t mxf4_instruction(int m, int n, int half)
{
    return 1u << 7 | 1u << 10 | (uint32_t)(n >> 3) << 17 | 1u << 23 | (uint32_t)(m >> 7) << 27 | (uint32_t)(half * 2) << 4 |
           (uint32_t)(half * 2) << 29;
}

// 64 columns of both operands; accumulates onto D if `onto`.
template <int CTAS> __device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t scale_a,
                                                             uint32_t scale_b, bool onto)
{
    if constexpr (CTAS == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(instruction), "r"(scale_a), "r"(scale_b), "r"((uint32_t)onto) : "memory");
    else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(instruction), "r"(scale_a), "r"(scale_b), "r"((uint32_t)onto) : "memory");
}

}  // namespace uq
