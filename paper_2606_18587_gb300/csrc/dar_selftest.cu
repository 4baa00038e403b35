// dar_selftest.cu -- dar_check_bounded_wait: exercises the give-up path that
// every kernel of the library shares when a bounded wait runs out (report
// DAR_ERR_DEVICE, let the block's own copies land, release tensor memory,
// exit), on a barrier that nothing ever completes; and that a warp has one
// verdict on a wait that only some of its lanes have given up.
#include "dar_common.cuh"
#include "dar_launch.h"
#include "dar_sm100.cuh"

namespace dar {
namespace {

constexpr unsigned kCopyBytes = 256;
constexpr uint32_t kTmemCols = 32;  // the smallest allocation

static __device__ __align__(128) unsigned char g_copy_src[kCopyBytes];

__global__ void __launch_bounds__(96, 1) bounded_wait_check_kernel(int32_t *status, unsigned long long limit_ns)
{
    using namespace sm100;
    __shared__ __align__(128) unsigned char buf[kCopyBytes];
    // [0]: the copy landed; [1]: never completed; [2]: completed when half of warp 2 has given up
    __shared__ __align__(8) uint64_t bars[3];
    __shared__ uint32_t tmem_slot;
    __shared__ int ran_out;
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        mbar_init(&bars[0], 1);
        mbar_init(&bars[1], 1);
        mbar_init(&bars[2], 1);
        ran_out = 0;
        mbar_init_fence();
    }
    if (warp == 1) {
        tmem_alloc(&tmem_slot, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    unsigned passed = 0;
    if (warp == 2)
        passed = __ballot_sync(0xffffffffu, mbar_wait_warp(&bars[2], 0, nullptr,
                                                           threadIdx.x % 32 < 16 ? limit_ns : kWaitLimitNs));
    if (threadIdx.x == 0) {
        // a copy of this block in flight when the wait gives up
        mbar_expect_tx(&bars[0], kCopyBytes);
        bulk_g2s(buf, g_copy_src, kCopyBytes, &bars[0]);
        // nothing arrives on bars[1]: this wait runs out after limit_ns
        if (!mbar_wait(&bars[1], 0, nullptr, limit_ns)) {
            ran_out = 1;
            // the give-up path: own copies land (bounded) before the block leaves
            mbar_wait(&bars[0], 0, nullptr);
        }
        // half of warp 2 has given up by then: its wait began with this one, and limits are looked at every 160 us
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < limit_ns + 1000000ull)
            __nanosleep(1000);
        mbar_arrive(&bars[2]);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 64 && ran_out && passed == 0u)
        report(status, DAR_ERR_DEVICE);
    if (warp == 1)
        tmem_dealloc(tmem, kTmemCols);
}

}  // namespace
}  // namespace dar

extern "C" dar_status dar_check_bounded_wait(int32_t *status, uint32_t limit_us, void *stream)
{
    if (!status || limit_us < 1 || limit_us > 2000000u) {
        dar::set_last_error("dar_check_bounded_wait: status must be non-NULL and limit_us in [1, 2000000]");
        return DAR_ERR_INVALID_ARG;
    }
    dar::bounded_wait_check_kernel<<<1, 96, 0, static_cast<cudaStream_t>(stream)>>>(
        status, (unsigned long long)limit_us * 1000ull);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) {
        dar::set_last_error(cudaGetErrorString(e));
        return DAR_ERR_CUDA;
    }
    dar::set_last_error("");
    return DAR_OK;
}
