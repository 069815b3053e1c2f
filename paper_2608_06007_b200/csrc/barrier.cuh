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

// As barrier_passed, but the warp may be set aside for a microsecond.
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
    return done != 0;
}

// Waits for the phase of that parity to end; false when it does not within about a second, or as many as spins / kWaitSpins.
// ROLLED: the loop is not unrolled, for kernels that wait in many places and whose code should be short.
constexpr uint32_t kWaitSpins = 1u << 20;
template <bool ROLLED = false>
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, uint32_t spins = kWaitSpins)
{
    if (barrier_passed(bar, parity)) return true;
    if constexpr (ROLLED) {
#pragma unroll 1
        for (uint32_t spin = 0; spin < spins; spin++) {
            if (barrier_try(bar, parity)) return true;
            if (spin > 64) __nanosleep(500);
        }
    } else {
        for (uint32_t spin = 0; spin < spins; spin++) {
            if (barrier_try(bar, parity)) return true;
            if (spin > 64) __nanosleep(500);
        }
    }
    return false;
}

}  // namespace tc
