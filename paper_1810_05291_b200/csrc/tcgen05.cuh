// The instructions of the matrix unit, its memory and its copies, one wrapper each, and bounded
// waits on shared-memory barriers.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace ss {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// The same address in block `rank` of the cluster.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// An arrival at a barrier of either block of a pair (an address from cluster_addr). It releases to
// this block only, which is all that operands in shared memory need: their stores are complete, and
// visible to the matrix unit, once the fence of smem_to_async has passed. A release to the cluster
// would wait for every load that the thread has under way.
__device__ __forceinline__ void mbar_arrive_pair(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

// Waits until the phase of that parity has completed. Gives up, returns false and raises *abort
// after a number of tries that no working launch comes near (a try suspends for a while by
// itself), or when another thread of the block has given up.
constexpr int kMaxTries = 1 << 20;
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort, int tries = kMaxTries) {
#pragma unroll 1
    for (int i = 0; i < tries; ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 63) == 63 && *abort != 0) return false;
    }
    *abort = 1;
    return false;
}

// The same for a warp whose control flow has to stay uniform: gives no answer. When it gave up, or
// *abort was up before, its caller goes on; further waits of the block end at once.
__device__ __forceinline__ void mbar_wait_uniform(uint32_t bar, uint32_t parity, const int* abort) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .u32 n, f;\n\tmov.u32 n, 0;\n"
        "TRY:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%0], %1;\n\t@p bra DONE;\n\t"
        "ld.volatile.shared.u32 f, [%2];\n\tsetp.ne.u32 p, f, 0;\n\t@p bra DONE;\n\t"
        "add.u32 n, n, 1;\n\tsetp.lt.u32 p, n, %3;\n\t@p bra TRY;\n\t"
        "st.volatile.shared.u32 [%2], 1;\n"
        "DONE:\n\t}"
        ::"r"(bar), "r"(parity), "r"(smem_addr(abort)), "n"(kMaxTries) : "memory");
}

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

__device__ __forceinline__ void mbar_init_visible() {  // to the copies and the matrix unit too
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// Shared memory written by ordinary stores, before the matrix unit reads it.
__device__ __forceinline__ void smem_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A box of a tensor to this block's shared memory; its bytes are counted by the barrier at `bar` of
// either block of a pair (an address from cluster_addr).
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const void* map, uint32_t bar, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}

// A box of a matrix to this block's shared memory.
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* map, uint32_t bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}

// Untiled copy: addresses and size in multiples of 16 bytes.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bar, uint32_t bytes) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %3, [%2];"
                 ::"r"(dst), "l"(__cvta_generic_to_global(src)), "r"(bar), "r"(bytes) : "memory");
}

// Tensor memory of a pair of blocks: one warp of each calls these.
__device__ __forceinline__ void tmem_alloc_pair(uint32_t dst, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t addr, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// D[tmem] (+)= A B over a pair of blocks, both operands bf16 in shared memory: each block holds
// half of A's rows (and of D's) and half of B's columns. Issued by one thread of the first block.
__device__ __forceinline__ void tc_mma_bf16_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
// Arrives at `bar` of both blocks when every matrix instruction issued so far by this thread has finished.
__device__ __forceinline__ void tc_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
}

// 32 columns of a warp's 32 lanes.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory operand whose contraction index is the slow one: panels of 64 elements (128
// bytes, swizzled in units of 16 bytes) by rows of the contraction index; `panel` bytes from one
// panel to the next, 1024 from 8 rows to the next 8.
__device__ __forceinline__ uint64_t tc_desc_rows(uint32_t addr, uint32_t panel) {
    return static_cast<uint64_t>((addr >> 4) & 0x3FFF) | (static_cast<uint64_t>((panel >> 4) & 0x3FFF) << 16) |
           (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// fp32 sums of bf16 products, both operands with the contraction index slow.
__device__ __forceinline__ constexpr uint32_t tc_idesc_bf16_rows(uint32_t m, uint32_t n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((n >> 3) << 17) | ((m >> 4) << 24);
}

}  // namespace ss
