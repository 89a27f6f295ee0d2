// async.cuh -- barriers in shared memory that asynchronous copies report to,
// with waits that end.
#pragma once

#include <stdint.h>

namespace av {

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

constexpr uint64_t kGiveUpNs = 4000000000ull;

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// Waits for the barrier's phase; false after some seconds, or at once when the
// block has given up elsewhere (*dead, in shared memory).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t phase, volatile int *dead)
{
    uint64_t began = 0;
    for (uint32_t spins = 0;; ++spins) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                     "selp.b32 %0, 1, 0, p;\n\t}"
                     : "=r"(done)
                     : "r"(bar), "r"(phase)
                     : "memory");
        if (done)
            return true;
        if ((spins & 63) != 63)
            continue;
        if (*dead)
            return false;
        const uint64_t t = now_ns();
        if (!began)
            began = t;
        else if (t - began > kGiveUpNs) {
            *dead = 1;
            return false;
        }
    }
}

// A block that gave up leaves copies still under way some time to land.
__device__ __forceinline__ void linger()
{
    const uint64_t began = now_ns();
    while (now_ns() - began < 10000000ull) {
    }
}

// `bytes` from global to shared memory, both and their number multiples of 16;
// counted at the barrier.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

}  // namespace av
