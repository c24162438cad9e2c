// Fifth-generation tensor core instructions (tcgen05), tensor copies and waits bounded in time, as thin wrappers.
#pragma once

#include "sgd_common.cuh"

namespace zipml {

constexpr unsigned long long kTcWaitNs = 2000000000ull;       // a wait that takes longer gives up
constexpr unsigned long long kTcSettleNs = 20000000ull;

__device__ __forceinline__ unsigned long long global_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

// Waits for a phase of a shared-memory barrier; false, with ZIPML_ERR_TIMEOUT recorded, after `limit`, or once another thread
// of the block has given up.  Two warps that wait for the same thing may get different answers, if one gives up just before it comes: what they
// do together afterwards (a barrier that wants all of them) needs tc_agree first.
static __device__ __noinline__ bool tc_wait_long(uint64_t* bar, uint32_t parity, volatile int* gave_up, DeviceStatus* status, int where, unsigned long long limit) {
    const unsigned long long began = global_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        if (*gave_up) return false;
        if (global_ns() - began > limit) break;
    }
    *gave_up = 1;
    set_status(status, ZIPML_ERR_TIMEOUT, where);
    return false;
}
__device__ __forceinline__ bool tc_wait(uint64_t* bar, uint32_t parity, volatile int* gave_up, DeviceStatus* status, int where,
                                        unsigned long long limit = kTcWaitNs) {
    return mbar_try_wait(bar, parity) || tc_wait_long(bar, parity, gave_up, status, where, limit);
}
// Whether all `threads` threads that share the named barrier say yes; each of them comes here, whatever its waits have said.
__device__ __forceinline__ bool tc_agree(bool yes, int barrier, int threads) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"((uint32_t)yes), "r"(barrier), "r"(threads) : "memory");
    return all != 0;
}
// For a block that has given up, between its last copy or product and the end of the memory these may still be at: they take microseconds.
static __device__ __noinline__ void tc_settle() {
    const unsigned long long began = global_ns();
    while (global_ns() - began < kTcSettleNs) __nanosleep(1000);
}

// The same address in CTA `rank` of the cluster, and an arrival there.  Its release has the default scope, a CTA's: that the products which the
// other CTA issues then see what this one has stored to its own shared memory is an assumption about the hardware, which reads each CTA's half
// where it lies, and not a guarantee of the memory model.  (With .release.cluster, which would be one, an arrival took 2,000 cycles.)
__device__ __forceinline__ uint32_t tc_peer(const void* p, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void tc_arrive_at(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// A tensor copy into this CTA's shared memory whose bytes count on a barrier of the pair's (its own or the other CTA's).
__device__ __forceinline__ void tc_copy_2d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_copy_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar)) : "memory");
}

// Shared-memory operand with the 128-byte swizzle.  Depth-major (K): rows of 128 bytes, 8 of them `sbo` apart.  Row-major (MN): 64
// values of the outer dimension are 128 bytes, the next 64 `lbo` on, 8 of the depth `sbo` apart.
__device__ __forceinline__ uint64_t tc_operand(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// 16-bit operands (both bf16 or both fp16), fp32 sums, m x n x 16 (m 128, or 256 for a pair of CTAs); `a_outer`: A is stored row-major (MN).
__host__ __device__ constexpr uint32_t tc_kind(bool bf16, bool a_outer, int m, int n) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (a_outer ? 1u << 15 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// D += A B.  PAIR: issued by the pair's first CTA for both; each holds 128 rows of A and of D and half of B's n.
template <bool PAIR>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool accumulate) {
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"((uint32_t)accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"((uint32_t)accumulate) : "memory");
}
// One lane of a converged warp, chosen so that the compiler sees a uniform branch: what a matrix instruction takes then stays in uniform
// registers.  (An `if (lane == 0)` around the loop cost some 100 cycles an instruction in moves.)
__device__ __forceinline__ bool tc_elect() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
// Arrives on `bar` (PAIR: at that place in both CTAs) once every product issued so far by this thread has ended.
template <bool PAIR>
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tc_alloc(uint32_t* slot, uint32_t columns) {
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tc_free(uint32_t tmem, uint32_t columns) {
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Makes this thread's ordinary shared-memory stores visible to the tensor cores and the copy engine.
__device__ __forceinline__ void tc_publish() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 16 columns of this warp's 32 lanes of tensor memory.
__device__ __forceinline__ void tc_load16(uint32_t tmem, uint32_t (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(tmem));
}
__device__ __forceinline__ void tc_load8(uint32_t tmem, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(tmem));
}
__device__ __forceinline__ void tc_store16(uint32_t tmem, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
                   "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(tmem)
                 : "memory");
}
__device__ __forceinline__ void tc_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

}  // namespace zipml
