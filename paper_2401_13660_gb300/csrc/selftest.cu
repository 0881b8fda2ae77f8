// Diagnostic of the library's bounded device-side waits (failure detection).
// Every wait in the kernels goes through mbar_wait_for: when the awaited
// phase does not complete within its limit the kernel records MB_ERR_TIMEOUT
// in the caller's status block and returns, instead of hanging the GPU. This
// kernel makes that path run on purpose, as a group of four warps goes it: the
// first waits on an mbarrier that nothing arrives on, for a caller-chosen
// number of SM clocks, gives up and then arrives there itself, so that the
// others see the phase complete. All four must give up with it (group_all): a
// warp that went on would wait for the first at the group's own barrier, which
// has no limit. Here they count themselves instead. The first one's timeout is
// recorded (detail = clocks waited) and the kernel exits with no copies in
// flight, so the context stays usable.
#include "common.cuh"
#include "tma.cuh"

namespace mbscan {
namespace {

__global__ void __launch_bounds__(128) wait_timeout_kernel(StatusBlock *sb, long long limit) {
    __shared__ uint64_t bar;
    __shared__ int left;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        mbar_init(&bar, 1);
        fence_mbar_init();
        left = 0;
    }
    __syncthreads();
    const long long t0 = clock64();
    const bool seen = __all_sync(kFull, mbar_wait_for(&bar, 0, warp == 0 ? limit : limit + kWaitCycles));
    const long long waited = clock64() - t0;
    if (threadIdx.x == 0) mbar_arrive(&bar);
    if (!group_all(1, seen) && lane == 0) atomicAdd(&left, 1);
    __syncthreads();
    if (threadIdx.x == 0) report(sb, left == 4 ? 4 /* MB_ERR_TIMEOUT */ : 3 /* MB_ERR_CUDA */, waited);
}

}  // namespace

cudaError_t launch_wait_timeout(StatusBlock *sb, long long limit, cudaStream_t s) {
    wait_timeout_kernel<<<1, 128, 0, s>>>(sb, limit);
    return cudaGetLastError();
}

}  // namespace mbscan
