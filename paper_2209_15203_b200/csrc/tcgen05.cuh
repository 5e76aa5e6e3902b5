// Thin wrappers of the sm_100a instructions the cross-entropy kernel is built from: mbarriers with bounded
// waits, TMA tile copies, tensor memory and the fifth-generation matrix instructions.
#pragma once

#include <cuda.h>

#include "train.cuh"

namespace tk {

__device__ __forceinline__ u32 smem_addr(const void* p) { return (u32)__cvta_generic_to_shared(p); }

// ---- mbarriers ----
__device__ __forceinline__ void mbar_init(u32 bar, u32 count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(u32 bar, u32 bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// `bar` is a shared::cluster address (mapped_addr), of this CTA or of its pair.  Nothing but the order of tensor memory
// accesses hangs on it, which tcgen05.fence keeps; a release at cluster scope would wait for every store
// the thread has in flight.
__device__ __forceinline__ void mbar_arrive_cluster(u32 bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// The hint lets the hardware hold the thread until the phase ends (or 1 ms has passed) instead of returning to poll: the loss of
// 8192 x 50257 x 768 took 407 us with it and 459 us without.
__device__ __forceinline__ bool mbar_try(u32 bar, u32 parity) {
    u32 done;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 1000000;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}
// Waits for the phase of the given parity to end, for about two seconds at most: every wait of the kernel is for
// work that takes microseconds, so running out means a fault elsewhere, and the caller leaves its loop.
constexpr long long kWaitCycles = 4000000000ll;
__device__ __forceinline__ bool mbar_wait(u32 bar, u32 parity) {
    if (mbar_try(bar, parity)) return true;
    const long long start = clock64();
    while (!mbar_try(bar, parity))
        if (clock64() - start > kWaitCycles) return false;
    return true;
}
__device__ __forceinline__ void mbar_init_fence() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

// ---- clusters of one or two CTAs ----
__device__ __forceinline__ u32 cluster_rank() {
    u32 r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ u32 mapped_addr(u32 addr, u32 rank) {
    u32 r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- TMA ----
// CG 2: the barrier may lie in the other CTA of the pair (both copies of a stage report to the leader's).
template <int CG>
__device__ __forceinline__ void tma_load(u32 dst, const CUtensorMap* map, u32 bar, int x, int y, int z) {
    if (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
            "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], "
            "[%2];" ::"r"(dst),
            "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
            : "memory");
}
template <int CG>
__device__ __forceinline__ void tma_load4(u32 dst, const CUtensorMap* map, u32 bar, int x, int y, int z, int u) {
    if (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], "
            "[%2];" ::"r"(dst),
            "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(u)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, "
            "%6}], [%2];" ::"r"(dst),
            "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(u)
            : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, u32 src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src),
                 "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void tma_store_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void tma_store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void smem_to_async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory ----
template <int CG> __device__ __forceinline__ void tmem_alloc(u32 dst_smem, u32 columns) {
    if (CG == 1)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(columns) : "memory");
}
template <int CG> __device__ __forceinline__ void tmem_free(u32 addr, u32 columns) {
    if (CG == 1) {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
    } else {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
    }
}
__device__ __forceinline__ void tcgen05_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// 32 columns of this warp's 32 lanes, one row per thread
__device__ __forceinline__ void tmem_load32(u32 addr, float (&v)[32]) {
    u32* r = (u32*)v;
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}

// ---- matrix instructions ----
// Shared-memory descriptor of an operand tile in the 128-byte swizzle: 1024-byte atoms of 8 rows x 128 bytes.
// K-major: rows are M (or N), 64 values of K each; `stride` leads to the next 8 rows, `lead` is not used.
// MN-major: rows are K, 64 values of M (or N) each; `stride` leads to the next 8 of K, `lead` to the next
// 64 of M (or N).
__device__ __forceinline__ u64 smem_desc(u32 addr, u32 lead, u32 stride) {
    return (u64)((addr >> 4) & 0x3fff) | (u64)((lead >> 4) & 0x3fff) << 16 | (u64)((stride >> 4) & 0x3fff) << 32 | (u64)1 << 46 |
           (u64)2 << 61;
}
// Instruction descriptor: bf16 operands, fp32 accumulators
__device__ __forceinline__ u32 mma_desc(int m, int n, bool a_mn, bool b_mn) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (u32)(n >> 3) << 17 | (u32)(m >> 4) << 24;
}
template <int CG>
__device__ __forceinline__ void mma_bf16(u32 tmem, u64 a, u64 b, u32 desc, bool accumulate) {
    u32 acc = accumulate;
    if (CG == 1)
        asm volatile(
            "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(tmem),
            "l"(a), "l"(b), "r"(desc), "r"(acc)
            : "memory");
    else
        asm volatile(
            "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(tmem),
            "l"(a), "l"(b), "r"(desc), "r"(acc)
            : "memory");
}
// Arrive on `bar` (with CG 2: on that barrier of both CTAs) when the matrix instructions issued so far are done
template <int CG> __device__ __forceinline__ void mma_commit(u32 bar) {
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
}

}  // namespace tk
