// The 5th-generation tensor cores from PTX: barriers with bounded waits, tensor memory, descriptors, products.
#pragma once

#include <cuda.h>

#include "afx_common.cuh"

namespace afx {

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// ---- mbarriers

__device__ __forceinline__ void mbar_init(uint64_t* bar, int arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// an arrival that also announces `bytes` of tensor copies
__device__ __forceinline__ void mbar_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.release.cta.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// a box of a four-dimensional tensor into shared memory
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
// Nanoseconds that a wait lasts at most (a build for tests may say otherwise).
#ifndef AFX_WAIT_NS
#define AFX_WAIT_NS 2000000000ull
#endif
// What the waits of a block share, in shared memory.
struct Patience {
    int gave_up;    // a waiter has
    uint32_t told;  // when one who works for long while others wait has last said that it goes on
};
__device__ __forceinline__ uint32_t nanoseconds() {
    uint32_t t;
    asm volatile("mov.u32 %0, %globaltimer_lo;" : "=r"(t));
    return t;
}
// Waits for the phase of that parity, but not for ever: false when another waiter of the block has given up, or after two
// seconds in which nobody said that it goes on, which no wait of a working kernel comes near.  (The clock's low word
// comes round after 4.3 s: both ages are seen above the limit in one look at least of those until then.  The first try stands
// in front of the loop, and there are no 64-bit times in it: 918 us for 8192 new tokens of 64 / 8 heads, 930 to 980 otherwise.)
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, volatile Patience* shared) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint32_t t0 = nanoseconds();
#pragma unroll 1
    while (!mbar_try_wait(bar, parity)) {
        // (a word that is written while it is read may be younger than the clock's reading: a millisecond more, so that no age is negative)
        const uint32_t told = shared->told, t = nanoseconds();
        if (shared->gave_up != 0) return false;
        if (min(t - t0, t - told + (1u << 20)) > static_cast<uint32_t>(AFX_WAIT_NS)) {
            shared->gave_up = 1;
            return false;
        }
    }
    return true;
}
// The wait of a thread that has given up for what it still has under way, which comes in any case: two seconds whatever the limit above.
__device__ __forceinline__ void mbar_drain(uint64_t* bar, uint32_t parity) {
    const uint32_t t0 = nanoseconds();
#pragma unroll 1
    while (!mbar_try_wait(bar, parity))
        if (nanoseconds() - t0 > 2000000000u) return;
}

__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- cluster launch control

// Asks to take over a block of this grid that has not begun; the 16-byte answer arrives with the barrier.
__device__ __forceinline__ void clc_ask(uint4* answer, uint64_t* bar) {
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)),
                 "r"(smem_u32(bar))
                 : "memory");
}
// The block's index in x; -1: refused, or there was none.
__device__ __forceinline__ int clc_place(const uint4* answer) {
    uint32_t taken, x;
    uint64_t lo, hi;
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(lo), "=l"(hi) : "r"(smem_u32(answer)) : "memory");
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        ".reg .b128 h;\n"
        "mov.b128 h, {%2, %3};\n"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "mov.u32 %1, 0;\n"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, h;\n"
        "}\n"
        : "=&r"(taken), "=&r"(x)
        : "l"(lo), "l"(hi));
    return taken != 0 ? static_cast<int>(x) : -1;
}

// ---- tensor memory

__device__ __forceinline__ void tmem_alloc(uint32_t* out, int columns) {  // one whole warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(out)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t at, int columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of the lane's row
__device__ __forceinline__ void tmem_ld32(float* r, uint32_t at) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
          "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]),
          "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]),
          "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(float* r, uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
                   "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

// ---- products

// Operand in shared memory with the 128-byte swizzle (16-byte piece c of row r at piece c ^ (r & 7) of its 128 bytes, groups
// of 8 rows 1024 bytes apart, base on 1024 bytes): the low word of its descriptor, which holds the place, and the high one.
// lead: bytes from one 128-byte-wide block to the next, where the operand's contiguous axis is not the one that is
// summed over (ignored otherwise).  A place x bytes further on is x / 16 more in the low word.
__device__ __forceinline__ uint32_t smem_desc(uint32_t at, uint32_t lead) { return ((at & 0x3FFFFu) >> 4) | ((lead >> 4) << 16); }
constexpr uint32_t kSmemDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);  // group stride, version of sm_100, 128-byte swizzle

// fp32 accumulator, 16-bit operands of one type, A with the summed axis contiguous; b_mn: B's other axis is contiguous.
__device__ __forceinline__ constexpr uint32_t mma_desc(bool bf16, int m, int n, bool b_mn) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) |
           (static_cast<uint32_t>(m >> 4) << 24);
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t is;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "elect.sync _|p, 0xFFFFFFFF;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(is));
    return is != 0;
}
// D[tmem] (+)= A[smem] B[smem], 16 of the summed axis.  (The operands' places are values that all lanes of the warp
// share: the instruction takes them from uniform registers.)
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        ".reg .b64 x, y;\n"
        "setp.ne.b32 p, %5, 0;\n"
        "mov.b64 x, {%1, %4};\n"
        "mov.b64 y, {%2, %4};\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n"
        "}\n" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(kSmemDescHigh), "r"(static_cast<uint32_t>(add))
        : "memory");
}
// D[tmem] (+)= A[tmem] B[smem]
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        ".reg .b64 y;\n"
        "setp.ne.b32 p, %5, 0;\n"
        "mov.b64 y, {%2, %4};\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n"
        "}\n" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(kSmemDescHigh), "r"(static_cast<uint32_t>(add))
        : "memory");
}
// The barrier gets an arrival when every product issued by this thread so far is done.
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

}  // namespace afx
