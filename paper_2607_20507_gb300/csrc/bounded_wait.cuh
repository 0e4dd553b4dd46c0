// bounded_wait.cuh -- mbarrier waits of a block's roles that give up together.
//
// A wait that has lasted for about a second raises the block's flag (dead) and sets
// CS_DEVICE_WAIT_TIMEOUT in the status word; while the flag is up every wait returns
// at once.
#pragma once

#include "cachespec.h"
#include "cs_device.cuh"

namespace cs {

constexpr long long kTcPatience = 2000000000;      // cycles: a second or so

// Waits for the phase of the given parity, asleep for up to 20 us.
__device__ __forceinline__ bool tc_asleep(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}\n"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
// Out of line, for the loop's code is long.  (try_wait sleeps for some 150 cycles at
// most, whatever it is told: between looks at the clock, 64 of them.)
inline __device__ __noinline__ void tc_wait_long(uint64_t* bar, uint32_t parity, volatile int* dead, int* status) {
    const long long t0 = clock64();
    while (!*dead) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (tc_asleep(bar, parity)) return;
        if (clock64() - t0 > kTcPatience) {
            *dead = 1;
            atomicOr(status, CS_DEVICE_WAIT_TIMEOUT);
        }
    }
}
__device__ __forceinline__ void tc_wait(uint64_t* bar, uint32_t parity, volatile int* dead, int* status) {
    if (!tc_asleep(bar, parity)) tc_wait_long(bar, parity, dead, status);
}
// Whether no wait has given up, the same answer in the whole warp.
__device__ __forceinline__ bool alive(volatile int* dead) { return !__any_sync(0xffffffffu, *dead); }

}  // namespace cs
