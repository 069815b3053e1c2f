// Device helpers that the kernels of tc_attn_decode share.
#pragma once

#include <type_traits>

#include "attn.h"
#include "ops_device.cuh"

namespace tc {

__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src, bool there)
{
    // nothing is read where `there` is false: 16 zero bytes are written
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_async4(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The kernels of one call overlap at their ends: allow_next lets the next one be launched once every CTA of
// this one has started, await_last waits until the one before is done and its writes are seen.
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void await_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

enum { kPlain = 0, kE4m3 = 1, kInt8 = 2 };

// Probabilities are multiplied by 2 to this power before they are rounded.  They are up to 2^8, since a running maximum may
// lag by that much; in fp16, whose normal numbers end at 2^-14, 2^7 more is what there is room for.  bf16 has room below, and
// values near 2^128, of which fp32 then holds sums of 2^16.
template <typename T> __device__ constexpr float probability_lift() { return std::is_same<T, __half>::value ? 7.f : -16.f; }

// Four codes as two pairs of fp16 numbers, exactly.
template <int KIND>
__device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    if constexpr (KIND == kE4m3) {
        lo = e4m3_to_half2(w), hi = e4m3_to_half2(w >> 16);
    } else {
        // int8: the bytes of 1024 + (code + 128), less 1152
        const uint32_t u = w ^ 0x80808080u, less = 0x64806480u;
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&less));
        const __half2 y = __hsub2(*reinterpret_cast<const __half2 *>(&b), *reinterpret_cast<const __half2 *>(&less));
        lo = *reinterpret_cast<const uint32_t *>(&x), hi = *reinterpret_cast<const uint32_t *>(&y);
    }
}
// Queries that meet codes are fp16 with a power of two taken out of each row, so that its largest finite
// magnitude `most` is in [2^14, 2^15).  The power to multiply with, and the one that undoes it.
__device__ __forceinline__ void query_powers(float most, float &up, float &down)
{
    const int e = most > 0.f ? max(static_cast<int>(__float_as_uint(most) >> 23) - 127, -100) : 14;
    up = __uint_as_float(static_cast<uint32_t>(14 - e + 127) << 23), down = __uint_as_float(static_cast<uint32_t>(e - 14 + 127) << 23);
}
__device__ __forceinline__ float2 query_pair(uint32_t w, bool bf16) { return bf16 ? unpack2<__nv_bfloat16>(w) : unpack2<__half>(w); }
__device__ __forceinline__ float finite_magnitude(float most, float2 f)
{
    if (fabsf(f.x) < INFINITY) most = fmaxf(most, fabsf(f.x));
    if (fabsf(f.y) < INFINITY) most = fmaxf(most, fabsf(f.y));
    return most;
}

// `follows`: a kernel of the same call was launched before this one, which then may start before that one's end.
template <typename Kernel>
int launch_attn(Kernel kernel, unsigned grid, unsigned threads, size_t shared, bool follows, const AttnParams &p, cudaStream_t s)
{
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(grid);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = shared;
    config.stream = s;
    cudaLaunchAttribute attribute{};
    attribute.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attribute.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &attribute;
    config.numAttrs = follows ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&config, kernel, p);
    return e == cudaSuccess ? TC_OK : cuda_fail(e, "kernel launch");
}

}  // namespace tc
