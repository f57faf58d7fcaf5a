// A pair of thread blocks on one tile: `tcgen05` with cta_group::2, TMA loads that report to the first block's mbarriers, TMA stores.
#pragma once
#include "pipe.cuh"

namespace aa {

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
// address of the same shared-memory place in another block of the cluster
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// One arrival of a warp whose lanes have all done their part, by its elected lane, on an mbarrier; CLUSTER: of a block of the cluster (a
// shared::cluster address).  It tells of tensor-memory reads, which are complete; a release at cluster scope would wait for the warp's global stores
// too (3000 cycles a tile).
template <bool CLUSTER> __device__ __forceinline__ void arrive_warp_e(uint32_t elected, uint32_t bar) {
    __syncwarp();
    if constexpr (CLUSTER)
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q mbarrier.arrive.shared::cluster.b64 _, [%0];\n\t}\n" ::"r"(bar), "r"(elected) : "memory");
    else
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}\n" ::"r"(bar), "r"(elected) : "memory");
}

// Tensor memory of both blocks: a warp of each calls these
template <uint32_t kCols> __device__ __forceinline__ void tmem_alloc_pair(uint32_t slot) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(slot), "n"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
}
template <uint32_t kCols> __device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(taddr), "n"(kCols) : "memory");
}
// Whether an mbarrier's phase is complete, without waiting
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// One lane of a warp in uniform control flow, chosen once: issues the instructions below.
__device__ __forceinline__ uint32_t elect_lane() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}\n" : "=r"(e));
    return e;
}
// D (+)= A B, one step of 16 of the sum.  PAIR: over both blocks of a pair (M = 256: 128 rows of A each, half of B's columns each), by the first.
#define AA_UMMA_STEP(group) "@q tcgen05.mma.cta_group::" group ".kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
template <bool PAIR> __device__ __forceinline__ void umma_step(uint32_t elected, uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %5, 0;\n\tsetp.ne.b32 p, %4, 0;\n\t" AA_UMMA_STEP("2") ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(elected) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %5, 0;\n\tsetp.ne.b32 p, %4, 0;\n\t" AA_UMMA_STEP("1") ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(elected) : "memory");
}
#undef AA_UMMA_STEP
// Four steps whose descriptors are kA and kB apart: 64 of the sum.  (As four separate instructions with an election each they took twice the
// time that the tensor cores need.)
#define AA_UMMA_FOUR(group)                                                                                  \
    "{\n\t.reg .pred p, q, t;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 q, %5, 0;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t" \
    "@q tcgen05.mma.cta_group::" group ".kind::f16 [%0], %1, %2, %3, p;\n\t"                                 \
    "add.s64 a, %1, %6;\n\tadd.s64 b, %2, %7;\n\t"                                                       \
    "@q tcgen05.mma.cta_group::" group ".kind::f16 [%0], a, b, %3, t;\n\t"                                   \
    "add.s64 a, a, %6;\n\tadd.s64 b, b, %7;\n\t"                                                         \
    "@q tcgen05.mma.cta_group::" group ".kind::f16 [%0], a, b, %3, t;\n\t"                                   \
    "add.s64 a, a, %6;\n\tadd.s64 b, b, %7;\n\t"                                                         \
    "@q tcgen05.mma.cta_group::" group ".kind::f16 [%0], a, b, %3, t;\n\t}\n"
template <bool PAIR, int kA, int kB> __device__ __forceinline__ void umma_four(uint32_t elected, uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
    if constexpr (PAIR) asm volatile(AA_UMMA_FOUR("2") ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(elected), "n"(kA), "n"(kB) : "memory");
    else asm volatile(AA_UMMA_FOUR("1") ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(elected), "n"(kA), "n"(kB) : "memory");
}
#undef AA_UMMA_FOUR
// Arrival once the instructions so far are complete: PAIR: at the mbarrier of both blocks
template <bool PAIR> __device__ __forceinline__ void umma_commit_e(uint32_t elected, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile(
            "{\n\t.reg .pred q;\n\t.reg .b16 m;\n\tsetp.ne.b32 q, %1, 0;\n\tmov.b16 m, 3;\n\t"
            "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}\n" ::"r"(bar), "r"(elected) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
            "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(bar), "r"(elected) : "memory");
}
// the same of a pair's instructions at an mbarrier of the first block alone
__device__ __forceinline__ void umma_commit_first(uint32_t elected, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(bar), "r"(elected) : "memory");
}
// 3-D tiled load into this block's memory by the elected lane of a warp in uniform control flow (every operand of a load inside an
// `if (lane == 0)` region takes a detour).  PAIR: it reports to an mbarrier of either block of the pair (a shared::cluster address).
template <bool PAIR> __device__ __forceinline__ void tma_load_3d_e(uint32_t elected, uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
            "@q cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}\n"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar), "r"(elected) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
            "@q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}\n"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar), "r"(elected) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory"); }
__device__ __forceinline__ void mbar_arrive_expect_tx_e(uint32_t elected, uint32_t bar, uint32_t bytes) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
        "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}\n" ::"r"(bar), "r"(bytes), "r"(elected) : "memory");
}

// 3-D tiled store of a staged box by the elected lane (what lies outside the tensor is left out); the groups of stores are a thread's own, so that a warp
// commits and waits as a whole
__device__ __forceinline__ void tma_store_3d_e(uint32_t elected, const CUtensorMap* map, int x, int y, int z, uint32_t src) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];\n\t}\n"
        ::"l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(src), "r"(elected) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;\n" ::: "memory"); }
// until all but the last N groups have been read out of shared memory
template <int N> __device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(N) : "memory"); }

}  // namespace aa
