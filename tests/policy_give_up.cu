// The policy loss with waits that give up as they would after two seconds, for test_gpu_policy_give_up.py:
// one warp's, from a given one on, at once, the others' after 20 ms; and with a current device of any
// number. All other code is the library's.
#include <cuda_runtime.h>

static int pretended = -1;
static cudaError_t device_now(int *device) {
    if (pretended < 0) return cudaGetDevice(device);
    *device = pretended;
    return cudaSuccess;
}
#define cudaGetDevice device_now
#include "blackwell.cuh"

namespace tmk {

struct Plan {
    int block, warp, after;
};
__device__ Plan plan = {-1, -1, 0};
constexpr int kMostThreads = 1 << 18;
__device__ unsigned waits[kMostThreads];  // of each thread

template <bool kCluster>
__device__ __forceinline__ bool planned_wait(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    if (!__isShared(const_cast<const int *>(gave_up))) return bar_wait_of<kCluster>(bar, parity, gave_up);  // for copies in flight
    const unsigned thread = blockIdx.x * blockDim.x + threadIdx.x;
    const unsigned n = thread < kMostThreads ? waits[thread]++ : 0;
    if (int(blockIdx.x) == plan.block && int(threadIdx.x >> 5) == plan.warp && n >= unsigned(plan.after)) {
        *gave_up = 1;
        return false;
    }
    const uint64_t t0 = global_ns();
    while (!(kCluster ? bar_try_cluster(bar, parity) : bar_try(bar, parity))) {
        if (*gave_up) return false;
        if (global_ns() - t0 > 20000000ull) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}

int set_error(int code, const char *) { return code; }

}  // namespace tmk

#define bar_wait planned_wait<false>
#define bar_wait_cluster planned_wait<true>
#include "policy.cu"

// What the library takes for the current device's number; -1: what it is.
extern "C" void pretend_device(int device) { pretended = device; }

// The warp whose waits give up from the one of number `after` on; block -1: none.
extern "C" int plan_give_up(int block, int warp, int after) {
    const tmk::Plan p = {block, warp, after};
    void *counts = nullptr;
    if (cudaGetSymbolAddress(&counts, tmk::waits) != cudaSuccess || cudaMemset(counts, 0, sizeof(tmk::waits)) != cudaSuccess) return 1;
    return cudaMemcpyToSymbol(tmk::plan, &p, sizeof p) != cudaSuccess;
}
