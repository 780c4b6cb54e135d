// Bounded waits on shared-memory mbarriers, shared by every kernel of the library that waits for a TMA copy or a
// tensor-core commit.  No wait in the library spins without a limit: after `cap` polls the waiting thread raises the
// CTA's abort flag (after which every wait of the CTA returns at once) and the context's device status word
// (kFlagTimeout, reported by fdkv_device_status as FDKV_ERR_TIMEOUT), and the kernel runs to its end without the data.
#pragma once

#include <cstdint>

#include "fdkv_internal.h"

namespace fdkv {

constexpr uint32_t kWaitCap = 1u << 22;  // polls before a wait gives up (0.4 s at 100 ns each, where a copy lands within microseconds)

__device__ __forceinline__ uint32_t mbar_try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}

// Waits for the phase with the given parity of the barrier at shared-memory address `bar`.
__device__ __forceinline__ void mbar_wait_bounded(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, int32_t* status,
                                                  uint32_t cap = kWaitCap) {
    if (mbar_try_wait(bar, parity)) return;  // the common case: one poll, no look at the abort flag
    if (*abort_flag) return;
    for (uint32_t i = 0; i < cap; ++i) {
        if (mbar_try_wait(bar, parity)) return;
        if ((i & 255u) == 255u && *abort_flag) return;
    }
    *abort_flag = 1;
    atomicMax(status, (int32_t)kFlagTimeout);
}

// Waits, a whole warp at a time, until a counter in shared memory has reached `target`.  One lane polls and sleeps in between: a plain load does not suspend the
// warp as a barrier's wait does, so that without the sleep the polls would take issue slots from the warps at work, and their limit would be up in a tenth of a second.
constexpr uint32_t kCountCap = 1u << 25;  // polls (8 s at 256 ns each: it may have to wait for a block's whole heads)
__device__ __forceinline__ void count_wait_bounded(const volatile uint32_t* count, uint32_t target, volatile uint32_t* abort_flag, int32_t* status,
                                                   uint32_t cap = kCountCap) {
    if ((threadIdx.x & 31) == 0) {
        uint32_t i = 0;
        while (*count < target && !*abort_flag) {
            if (i++ >= cap) {
                *abort_flag = 1;
                atomicMax(status, (int32_t)kFlagTimeout);
                break;
            }
            __nanosleep(100);
        }
    }
    __syncwarp();
}

}  // namespace fdkv
