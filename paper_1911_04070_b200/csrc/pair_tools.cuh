// Building blocks of the matrix-product kernels that run on pairs of CTAs (clusters of two, tcgen05 cta_group::2):
// one instruction multiplies a 256-row tile, each CTA holding 128 rows of A and half the columns of B in its own shared
// memory and 128 rows of the accumulator in its own tensor memory.  Against one CTA working alone this halves
// what every CTA has to read of B.  Loads are plain TMA tile loads (each CTA its own share), completion of both CTAs'
// loads is counted on a barrier of the pair's first CTA, whose thread issues the products.
#pragma once
#include <cuda_runtime.h>
#include <cstdint>

#include "tc5_tools.cuh"

namespace bpt {
namespace pair {

__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Every thread of both CTAs.
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, usable from this CTA, of the same shared-memory location in the pair's first CTA.
__device__ __forceinline__ uint32_t in_first(uint32_t saddr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(saddr));
    return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t mbar_cluster) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(mbar_cluster) : "memory");
}
// Bounded wait that also orders what the other CTA did before its arrival.  The clock is read every 32nd probe.
__device__ __forceinline__ bool wait_cluster(uint32_t mbar, uint32_t parity, long long limit = tc5::kWaitCycles) {
    long long start = 0;
    for (uint32_t it = 0;; ++it) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
                     : "=r"(ok) : "r"(mbar), "r"(parity) : "memory");
        if (ok) return true;
        if ((it & 31) == 31) {
            const long long now = clock64();
            if (start == 0) start = now;
            else if (now - start > limit) return false;
        }
    }
}
// Tile load into this CTA's shared memory, counted on a barrier of either CTA of the pair.
__device__ __forceinline__ void load_2d(uint32_t dst, const void* tmap, int c0, int c1, uint32_t mbar_cluster) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(tmap), "r"(c0), "r"(c1), "r"(mbar_cluster) : "memory");
}
// D (tensor memory of both CTAs) = A * B (+ D when acc != 0), 256 rows; issued by one thread of the first CTA.
__device__ __forceinline__ void mma(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t}\n"
                 :: "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(acc), "r"(tc5::desc_hi()) : "memory");
}
// Low descriptor word of an operand whose rows are the k index: 64-wide column blocks 8 KB apart (64 k rows of 128 bytes).
__device__ __forceinline__ uint32_t desc_lo_mn(uint32_t saddr) { return ((saddr >> 4) & 0x3fff) | ((8192u >> 4) << 16); }
// One arrival on the barrier at this offset in both CTAs once every product issued so far has completed.
__device__ __forceinline__ void commit_both(uint32_t mbar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 :: "r"(mbar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t slot_smem, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(slot_smem), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t taddr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(taddr), "r"(cols) : "memory");
}
// Tile stores from shared memory; rows and columns outside the tensor are not written.
__device__ __forceinline__ void store_2d(const void* tmap, int c0, int c1, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" :: "l"(tmap), "r"(c0), "r"(c1), "r"(src) : "memory");
}
__device__ __forceinline__ void store_3d(const void* tmap, int c0, int c1, int c2, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" :: "l"(tmap), "r"(c0), "r"(c1), "r"(c2), "r"(src) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// At most N of this thread's store groups still read their shared memory / are still under way at all.
template <int N> __device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" :: "n"(N) : "memory"); }
template <int N> __device__ __forceinline__ void store_wait() { asm volatile("cp.async.bulk.wait_group %0;" :: "n"(N) : "memory"); }

}  // namespace pair
}  // namespace bpt
