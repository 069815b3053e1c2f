// Barriers in shared memory, and waits on them that end.
#pragma once

#include <stdint.h>

namespace tc {

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool barrier_passed(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

// Waits for the phase of that parity to end; false when it does not within about a second.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity)
{
    if (barrier_passed(bar, parity)) return true;
    for (uint32_t spin = 0; spin < (1u << 20); spin++) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
        if (done) return true;
        if (spin > 64) __nanosleep(500);
    }
    return false;
}

}  // namespace tc
