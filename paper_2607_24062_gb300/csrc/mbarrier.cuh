// mbarrier helpers with time-bounded waits, shared by the tensor-core kernel
// and the wait self-test.  No wait here can spin forever: each gives up after
// a limit measured on %globaltimer.
#pragma once

#include <cstdint>

namespace acrl {
namespace {

constexpr uint64_t kWaitNs = 2000000000ull;  // 2 s: every legitimate wait is microseconds

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}

__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes)
                 : "memory");
}

__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}

__device__ __forceinline__ uint64_t global_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Wait for the completion of the phase of `bar` with parity `parity`.  Gives
// up after kWaitNs, or early once another role has set *abort (unless abort
// is null).
__device__ __forceinline__ bool wait_phase_inline(uint64_t* bar, uint32_t parity, volatile int32_t* abort,
                                                  uint64_t limit_ns = kWaitNs) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_ns();
    for (uint32_t i = 1;; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 255u) == 0u) {
            if (abort && *abort) return false;
            if (global_ns() - t0 > limit_ns) return false;
        }
    }
}

// The same as a call, for the places where it is rare: few instructions there, but what is live across it is spilled where
// it is more than a call preserves.
__device__ __noinline__ bool wait_phase(uint64_t* bar, uint32_t parity, volatile int32_t* abort,
                                        uint64_t limit_ns = kWaitNs) {
    return wait_phase_inline(bar, parity, abort, limit_ns);
}

}  // namespace
}  // namespace acrl
