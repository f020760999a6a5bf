// Shared-memory barriers (mbarrier) with bounded waits, for the kernels that feed the tensor cores.
#pragma once

#include <cstdint>

namespace scoot_dev {

constexpr unsigned long long kWaitNs = 2000000000ull;  // bounded waits give up after 2 s

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ unsigned long long global_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

__device__ __forceinline__ bool mbar_try(uint32_t addr, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(addr), "r"(parity)
        : "memory");
    return done;
}

// Whether the phase of the given parity has completed, at once.
__device__ __forceinline__ bool mbar_test(uint32_t addr, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(addr), "r"(parity)
        : "memory");
    return done;
}

// Whether three have, their latencies overlapped.
__device__ __forceinline__ bool mbar_test3(uint32_t a, uint32_t pa, uint32_t b, uint32_t pb, uint32_t c, uint32_t pc) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p, q, r;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 q, [%3], %4;\n\tmbarrier.test_wait.parity.shared::cta.b64 r, [%5], %6;\n\t"
        "and.pred p, p, q;\n\tand.pred p, p, r;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(a), "r"(pa), "r"(b), "r"(pb), "r"(c), "r"(pc)
        : "memory");
    return done;
}

// Waits (bounded) until the phase of the given parity of an mbarrier has
// completed; false if it gave up.  The clock is read only after a try that
// failed (which itself waits a while).
__device__ __forceinline__ bool mbar_wait(uint32_t addr, uint32_t parity) {
    if (mbar_try(addr, parity)) return true;
    const unsigned long long t0 = global_ns();
    while (!mbar_try(addr, parity))
        if (global_ns() - t0 > kWaitNs) return false;
    return true;
}

// The same bounded by the number of tries, each of which waits a microsecond at most (a few instructions, for kernels
// whose waits are on the way of everything): gives up after 0.1 to 4 s.  A test first: on a phase that
// has completed it takes 45 cycles, a try 115.
__device__ __forceinline__ bool mbar_wait_tries(uint32_t addr, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .u32 i;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t@p bra DONE;\n\t"
        "mov.u32 i, 4194304;\n"
        "AGAIN:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t@p bra DONE;\n\t"
        "add.u32 i, i, -1;\n\tsetp.ne.u32 q, i, 0;\n\t@q bra AGAIN;\n"
        "DONE:\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(addr), "r"(parity), "r"(1000u)
        : "memory");
    return done;
}

__device__ __forceinline__ void mbar_init(uint64_t* b, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count));
}

__device__ __forceinline__ void mbar_arrive_at(uint32_t addr) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* b) { mbar_arrive_at(smem_u32(b)); }

// Waits (bounded) for use u of a barrier that completes one phase per use.
__device__ __forceinline__ bool mbar_wait_use(uint64_t* b, int64_t u) { return mbar_wait(smem_u32(b), (uint32_t)(u & 1)); }

// The same for a whole warp, with one answer.
__device__ __forceinline__ bool warp_wait_use(uint64_t* b, int64_t u) {
    return __all_sync(0xffffffffu, mbar_wait_use(b, u));
}

// One arrival for a whole warp (an arrival per thread is an operation per thread on
// the barrier's word).
__device__ __forceinline__ void warp_arrive(uint64_t* b) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(b);
}

}  // namespace scoot_dev
