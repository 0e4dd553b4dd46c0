// selftest.cu -- the failure-detection self-test (cs_selftest_wait_timeout):
// the bounded mbarrier waits of the attention kernels, run on barriers that
// nothing arrives at.
#include "bounded_wait.cuh"
#include "cs_device.cuh"
#include "cs_internal.h"

namespace cs {

namespace {
// Two warps, a thread each, run the kernels' two bounded waits on barriers that
// nothing arrives at.  After about one second both give up; only if both have, and
// the second has raised its flag and said so, the first thread records
// CS_DEVICE_WAIT_TIMEOUT, as a kernel's role would.
__global__ void wait_selftest_kernel(int* status) {
    __shared__ uint64_t bar[2];
    __shared__ volatile int s_dead;
    __shared__ int s_status;
    bool gave_up = false;
    if (threadIdx.x == 0) {
        mbar_init(&bar[0], 1);
        mbar_init(&bar[1], 1);
        s_dead = 0;
        s_status = 0;
        fence_barrier_init();
    }
    __syncthreads();
    if (threadIdx.x == 0) gave_up = !mbar_wait_bounded(&bar[0], 0);
    if (threadIdx.x == 32) tc_wait(&bar[1], 0, &s_dead, &s_status);
    __syncthreads();
    if (gave_up && s_dead == 1 && s_status == CS_DEVICE_WAIT_TIMEOUT) atomicOr(status, CS_DEVICE_WAIT_TIMEOUT);
}
}  // namespace

cudaError_t launch_wait_selftest(int* status, cudaStream_t stream) {
    wait_selftest_kernel<<<1, 64, 0, stream>>>(status);
    return cudaGetLastError();
}

}  // namespace cs
