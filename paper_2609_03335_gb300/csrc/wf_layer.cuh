// What the calls on a layer's tensors share: the cache's addresses, division by
// the block size, conversions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "wf_internal.cuh"

// x / d for 0 <= x < 2^31 by a multiplication: m = ceil(2^(31 + l) / d) with l = ceil(log2 d) has an error of
// less than 2^l over 2^(31 + l) / d, so x * m is off by less than 2^(31 + l) / d, and the quotient is exact.
struct wf_div {
    uint32_t m, shift;
};

inline wf_div wf_make_div(uint32_t d)
{
    uint32_t l = 0;
    while ((1ull << l) < d) l++;
    return {(uint32_t)(((1ull << (31 + l)) + d - 1) / d), 31 + l};
}

__device__ __forceinline__ uint32_t wf_quot(uint32_t x, wf_div d) { return (uint32_t)(((uint64_t)x * d.m) >> d.shift); }

template <typename T> struct wf_pair;
template <> struct wf_pair<__half> {
    static __device__ __forceinline__ float2 to_float(uint32_t x) { return __half22float2(*reinterpret_cast<__half2 *>(&x)); }
    static __device__ __forceinline__ uint32_t of_float(float a, float b)
    {
        __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&h);
    }
};
template <> struct wf_pair<__nv_bfloat16> {
    static __device__ __forceinline__ float2 to_float(uint32_t x)
    {
        return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
    }
    static __device__ __forceinline__ uint32_t of_float(float a, float b)
    {
        __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&h);
    }
};

// Four E4M3 values (lowest byte first) as pairs of halves, which hold them exactly.
__device__ __forceinline__ uint2 wf_e4m3_halves(uint32_t x)
{
    uint2 r;
    asm("{ .reg .b16 lo, hi;\n"
        "  mov.b32 {lo, hi}, %2;\n"
        "  cvt.rn.f16x2.e4m3x2 %0, lo;\n"
        "  cvt.rn.f16x2.e4m3x2 %1, hi; }"
        : "=r"(r.x), "=r"(r.y) : "r"(x));
    return r;
}

// Rounded to nearest, even; beyond 448 to +-448; a in the lower byte.
__device__ __forceinline__ uint32_t wf_e4m3_of(float a, float b)
{
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
