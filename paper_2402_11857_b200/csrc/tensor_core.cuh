// 5th-generation tensor cores: descriptors, issue, completion and tensor memory, as used by one CTA.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace liec {

// A [K][64] block of 16-bit elements whose K rows of 128 bytes lie one after another, 16-byte chunk j of row t at place
// j ^ (t & 7): the 128-byte swizzle for an operand whose contiguous axis is not the product's.  Blocks of further 64
// elements follow `block_bytes` apart; groups of 8 rows, 1024 bytes.
__device__ __forceinline__ uint64_t tc_descriptor(uint32_t smem_address, uint32_t block_bytes) {
    return (uint64_t)((smem_address & 0x3ffffu) >> 4) | (uint64_t)(block_bytes >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ constexpr uint32_t tc_swizzled(int row, int chunk) { return (uint32_t)(row * 128 + ((chunk ^ (row & 7)) << 4)); }

// bfloat16 times bfloat16 into binary32, both operands with their contiguous axis along M and N.
__host__ __device__ constexpr uint32_t tc_instruction(int m, int n) {
    return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(n / 8) << 17 | (uint32_t)(m / 16) << 24;
}

// Products of a pair of CTAs (a cluster of two): each holds half of A's rows and of the accumulator's, and half of B's
// columns, at the same places of its memory; the first CTA issues.
__device__ __forceinline__ void tc_mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, bool add) {
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p; }"
                 ::"r"(d), "l"(a), "l"(b), "r"(instruction), "r"((uint32_t)add) : "memory");
}
// The barrier at this place in both CTAs gets one arrival when all products issued so far by this thread are done.
__device__ __forceinline__ void tc_commit_pair(uint32_t barrier) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(barrier), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// A whole warp of each CTA of the pair; the address is written to shared memory.
__device__ __forceinline__ void tc_alloc_pair(uint32_t where, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_free_pair(uint32_t tmem, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}

// 32 columns of this warp's 32 lanes; complete when it returns.
__device__ __forceinline__ void tc_load(uint32_t tmem, float (&v)[32]) {
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
                   "=r"(r[31])
                 : "r"(tmem)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// What the threads of this CTA wrote to shared memory becomes visible to copies and products.
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void barrier_init(uint32_t barrier, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(barrier), "r"(count) : "memory");
}
// Address of the same place in the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t in_cta(uint32_t address, int rank) {
    uint32_t to;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(address), "r"(rank));
    return to;
}
// An arrival at a barrier of the cluster.  Every one has to be waited for before the CTA that it goes to ends.  (What it
// announces are the arriving CTA's own shared memory, made visible to the products by async_fence, and tensor memory; a release
// for the whole cluster would wait for all earlier accesses to global memory as well, some 1500 cycles.)
__device__ __forceinline__ void barrier_arrive_cluster(uint32_t cluster_address) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_address) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t barrier, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(barrier), "r"(bytes) : "memory");
}
// True when the phase completed; polls at most `limit` times.
__device__ __forceinline__ bool barrier_wait(uint32_t barrier, uint32_t parity, uint32_t limit) {
    uint32_t done = 0;
    for (uint32_t spin = 0; spin < limit && !done; ++spin)
        asm volatile("{ .reg .pred q; mbarrier.try_wait.parity.shared::cta.b64 q, [%1], %2; selp.u32 %0, 1, 0, q; }"
                     : "=r"(done) : "r"(barrier), "r"(parity) : "memory");
    return done != 0;
}
// The same for a whole warp.
__device__ __forceinline__ bool barrier_wait_warp(uint32_t barrier, uint32_t parity, uint32_t limit) {
    return __all_sync(0xffffffffu, barrier_wait(barrier, parity, limit));
}
// True in one thread of a whole warp.  (Loops that a warp walks as one keep what they compute in uniform registers,
// which products and copies take their operands from: with a loop in one thread alone a stage's four products took 380
// cycles to issue.)
__device__ __forceinline__ bool elected() {
    uint32_t yes;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(yes));
    return yes != 0u;
}

// A box of a three-axis array into this CTA's shared memory; x times the element's size is a multiple of 16 bytes.
__device__ __forceinline__ void copy_box(uint32_t to, const void *map, int x, int y, int z, uint32_t barrier) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(z), "r"(barrier) : "memory");
}

}  // namespace liec
