// What kernels that copy asynchronously share: barriers in shared memory and bounded waits on them.
#pragma once

#include "qesgd_internal.h"

namespace {

constexpr uint64_t COARSE_TIMER_NS = 1024ull;        // limits below this mean "one look, then give up"

// ------------------------------------------------------------- primitives ----
__device__ __forceinline__ uint32_t smem_u32(const void *p)
{
    return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void mbar_init(uint64_t *bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)),
                 "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0u;
}
// Has a wait that began at t0 used up `limit`?  The global timer may tick as coarsely as a
// microsecond, so a smaller limit is read as "give up after one round of looks".
__device__ __forceinline__ bool expired(uint64_t t0, uint64_t limit)
{
    return limit < COARSE_TIMER_NS || now_ns() - t0 > limit;
}
// Bounded wait for phase `parity` of a barrier; gives up early when `*stop` is set.
__device__ __forceinline__ bool mbar_wait(uint64_t *bar, uint32_t parity, const volatile uint32_t *stop,
                                          uint64_t limit)
{
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = now_ns();
    for (;;) {
        for (int n = 0; n < 32; ++n)
            if (mbar_try_wait(bar, parity)) return true;
        if (*stop != 0u || expired(t0, limit)) return false;
    }
}

}  // namespace
