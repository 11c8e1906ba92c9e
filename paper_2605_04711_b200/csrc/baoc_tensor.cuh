// Device and host helpers of the matrix product: barriers in shared memory with bounded waits, tiled asynchronous copies, the
// tensor cores' descriptors and instructions (sm_100a), accumulators in tensor memory.
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "baoc_device.cuh"

namespace baoc {

// One lane of a converged warp, the same at every call.  Copies and products are issued under it by a warp whose lanes all go
// through the loop with the same values.  (Under a test of the lane's number a step of four products took 530 clocks of its issuing
// thread, whatever the tile, and bound the large ones: 16384 x 2048 into 8192 366 -> 346 us in a short row.  That the operands' way
// to where these instructions take them costs less this way is a guess; the times are not.)
__device__ __forceinline__ bool elected() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one;
}
__device__ __forceinline__ int uniform_warp() { return __shfl_sync(0xffffffffu, int(threadIdx.x >> 5), 0); }

// ---- barriers --------------------------------------------------------------------
// No wait is endless: one that takes longer than this reports false, and its caller gives the whole tile loop up.  (The longest
// work between two arrivals, 1024 steps of copies and products, takes under a millisecond.)
constexpr uint64_t kWaitNs = 10000000000ull;

__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// an address of this CTA's shared memory in that of another CTA of the cluster
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void bar_arrive_at(uint32_t bar, uint32_t rank) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(at_rank(bar, rank)) : "memory");
}
// (acquires at cluster scope: a pair's barriers are also arrived at from the other CTA)
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    if (bar_try(bar, parity)) return true;
    const uint64_t start = now_ns();
    for (uint32_t i = 0; i < 0xffffffffu; ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 63) == 63 && now_ns() - start > kWaitNs) return false;
    }
    return false;
}

// a whole warp's wait: its lanes agree
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, bar_wait(bar, parity)); }

// ---- tiled copies ----------------------------------------------------------------
// x (elements of the contiguous dimension) is a multiple of 64 bf16 everywhere: copies start on 128-byte boundaries of a row.
// kCtas = 2: bar may be that of the pair's first CTA (an address from at_rank).
template <int kCtas>
__device__ __forceinline__ void copy_tile(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (kCtas == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
// the way back: a box of shared memory to its place, rows and columns outside the matrix left out (x, y not negative)
__device__ __forceinline__ void store_tile(const CUtensorMap* map, uint32_t src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
template <int kPending>
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kPending) : "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void shared_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor cores ----------------------------------------------------------------
// Shared-memory operand of 128-byte rows with the 128-byte swizzle that the tiled copy writes.  K-major: rows of 64 k, groups of
// 8 rows 1024 bytes apart.  MN-major: rows of 64 m (or n), one row per k; groups of 8 k are 1024 bytes apart, the next 64 m
// follow after `lead` bytes.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lead) {
    return uint64_t((addr & 0x3ffff) >> 4) | uint64_t((lead & 0x3ffff) >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// bf16 x bf16 into fp32
__host__ __device__ constexpr uint32_t product_desc(int m, int n, bool a_mn, bool b_mn) {
    return 1u << 4 | 1u << 7 | 1u << 10 | uint32_t(a_mn) << 15 | uint32_t(b_mn) << 16 | uint32_t(n >> 3) << 17 | uint32_t(m >> 4) << 24;
}
template <int kCtas>
__device__ __forceinline__ void product(uint32_t acc, uint64_t a, uint64_t b, uint32_t desc, uint32_t add) {
    if constexpr (kCtas == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(acc), "l"(a), "l"(b), "r"(desc), "r"(add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(acc), "l"(a), "l"(b), "r"(desc), "r"(add) : "memory");
}
// the barrier (of both CTAs of a pair) is arrived at when the products issued so far are done
template <int kCtas>
__device__ __forceinline__ void product_commit(uint32_t bar) {
    if constexpr (kCtas == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(uint16_t(3)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int kCtas>
__device__ __forceinline__ void acc_alloc(uint32_t where, uint32_t columns) {         // a whole warp (of each CTA of a pair)
    if constexpr (kCtas == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <int kCtas>
__device__ __forceinline__ void acc_free(uint32_t acc, uint32_t columns) {
    if constexpr (kCtas == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(acc), "r"(columns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(acc), "r"(columns) : "memory");
}
__device__ __forceinline__ void acc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void acc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of a thread's row (its warp's quarter of the 128 lanes)
__device__ __forceinline__ void acc_load(uint32_t acc, float (&v)[32]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(acc));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// the same of 16 columns
__device__ __forceinline__ void acc_load(uint32_t acc, float (&v)[16]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(acc));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

}  // namespace baoc
