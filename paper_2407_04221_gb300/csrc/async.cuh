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

#ifndef AV_GIVE_UP_NS
#define AV_GIVE_UP_NS 4000000000ull
#endif
constexpr uint64_t kGiveUpNs = AV_GIVE_UP_NS;

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

// A chain of kernels of one call: each but the first may start while the one
// before it ends (its set-up under the other's last blocks), and touches memory
// only after `after_previous`, when that one has ended and its results are
// there.  `next_may_start` holds once all blocks have said it, so the next
// kernel takes no place that one of this kernel's blocks still needs.  It saves
// 2 us a kernel: the feed-forward's gradient, of 4,099 x 520 x 1,368, took 75.8
// us and takes 68.6, of 600 x 256 x 512 36.9 and 31.7.
__device__ __forceinline__ void after_previous()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("fence.proxy.async.global;" ::: "memory");  // (bulk copies read what it wrote)
}
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <class... P, class... A>
cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t shared, cudaStream_t st, bool chained, A... args)
{
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = block;
    config.dynamicSmemBytes = shared;
    config.stream = st;
    config.attrs = &attr;
    config.numAttrs = chained ? 1 : 0;
    return cudaLaunchKernelEx(&config, kernel, static_cast<P>(args)...);
}

}  // namespace av
