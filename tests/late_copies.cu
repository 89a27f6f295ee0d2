// late_copies.cu -- an operator's kernels (AV_SOURCE) whose waits end after 20
// ms, one of which waits for 16 bytes more than are on their way: those that
// the `nth` time thread 0 of block `block` announces.  Every copy lands.
#define AV_GIVE_UP_NS 20000000ull
#include "async.cuh"

namespace av {
__device__ int late_block, late_nth, late_calls;
__device__ uint32_t late()
{
    return threadIdx.x == 0 && (int)blockIdx.x == late_block && late_calls++ == late_nth ? 16u : 0u;
}
}  // namespace av

#define bar_expect(bar, bytes) bar_expect(bar, (bytes) + av::late())
#include AV_SOURCE
#undef bar_expect
#include "policy.cu"

extern "C" int set_late(int block, int nth)
{
    const int none = 0;
    cudaError_t e = cudaMemcpyToSymbol(av::late_block, &block, sizeof block);
    if (e == cudaSuccess)
        e = cudaMemcpyToSymbol(av::late_nth, &nth, sizeof nth);
    if (e == cudaSuccess)
        e = cudaMemcpyToSymbol(av::late_calls, &none, sizeof none);
    return (int)e;
}
