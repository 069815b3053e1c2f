// Device-side number formats and small helpers of the operators on a paged layer.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "ops.h"

namespace tc {

__device__ __forceinline__ uint32_t quick_div(uint32_t n, FastDiv f) { return (__umulhi(n, f.mul) + n) >> f.shift; }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Two floats rounded to 16 bits, a in the low half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

// Two floats as e4m3 codes (to nearest even), a in the low byte.
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b)
{
    uint16_t v;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(b), "f"(a));
    return v;
}
// Two e4m3 codes (low 16 bits of w) as fp16, exactly.
__device__ __forceinline__ uint32_t e4m3_to_half2(uint32_t w)
{
    uint32_t v;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v) : "h"(static_cast<uint16_t>(w)));
    return v;
}
__device__ __forceinline__ uint32_t int8_pair(float a, float b)
{
    return (static_cast<uint32_t>(__float2int_rn(a)) & 0xffu) | ((static_cast<uint32_t>(__float2int_rn(b)) & 0xffu) << 8);
}

// W words at p, in one access: 16-byte accesses are aligned to 16 bytes, 32-byte ones to 32.
template <int W> struct Words { uint32_t w[W]; };
template <int W>
__device__ __forceinline__ Words<W> load_words(const void *p)
{
    Words<W> r;
    static_assert(W == 1 || W == 2 || W == 4 || W == 8);
    if constexpr (W == 1) r.w[0] = *static_cast<const uint32_t *>(p);
    if constexpr (W == 2) asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(p));
    if constexpr (W == 4) asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p));
    if constexpr (W == 8)
        asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7]) : "l"(p));
    return r;
}
template <int W>
__device__ __forceinline__ void store_words(void *p, const Words<W> &r)
{
    static_assert(W == 2 || W == 4 || W == 8);
    if constexpr (W == 2) asm volatile("st.global.v2.b32 [%0], {%1,%2};" ::"l"(p), "r"(r.w[0]), "r"(r.w[1]) : "memory");
    if constexpr (W == 4) asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]) : "memory");
    if constexpr (W == 8)
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7])
                     : "memory");
}

// N numbers of type T at p (aligned to min(16, N * sizeof(T)) bytes) as floats.
template <typename T, int N>
__device__ __forceinline__ void load_floats(const void *p, float *x)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; i++) {
            const float4 v = static_cast<const float4 *>(p)[i];
            x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
        }
    } else {
        uint32_t w[N / 2];
        if constexpr (N == 8) {
            const uint4 v = *static_cast<const uint4 *>(p);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else {
            static_assert(N == 4);
            const uint2 v = *static_cast<const uint2 *>(p);
            w[0] = v.x, w[1] = v.y;
        }
#pragma unroll
        for (int i = 0; i < N / 2; i++) {
            const float2 f = unpack2<T>(w[i]);
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_floats(void *p, const float *x)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; i++) static_cast<float4 *>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    } else {
        static_assert(N == 8);
        *static_cast<uint4 *>(p) = make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
    }
}

}  // namespace tc
