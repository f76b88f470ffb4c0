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

// Elements that are no finite numbers, in a word of two or four: their topmost bits.  An exponent of all ones (in E4M3 with a mantissa of all ones) carries into it.
template <typename T> __device__ __forceinline__ uint32_t wf_unfit(uint32_t x);
template <> __device__ __forceinline__ uint32_t wf_unfit<__half>(uint32_t x) { return ((x & 0x7C007C00u) + 0x04000400u) & 0x80008000u; }
template <> __device__ __forceinline__ uint32_t wf_unfit<__nv_bfloat16>(uint32_t x) { return ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
template <> __device__ __forceinline__ uint32_t wf_unfit<__nv_fp8_e4m3>(uint32_t x) { return ((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

template <typename T> __device__ __forceinline__ uint32_t wf_unfit(const uint4 &x)
{
    return wf_unfit<T>(x.x) | wf_unfit<T>(x.y) | wf_unfit<T>(x.z) | wf_unfit<T>(x.w);
}

// The larger magnitude of both halves each; NaN stays.
template <typename T> __device__ __forceinline__ uint32_t wf_larger(uint32_t most, uint32_t x);
template <> __device__ __forceinline__ uint32_t wf_larger<__half>(uint32_t most, uint32_t x)
{
    const __half2 r = __hmax2_nan(*reinterpret_cast<__half2 *>(&most), __habs2(*reinterpret_cast<__half2 *>(&x)));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <> __device__ __forceinline__ uint32_t wf_larger<__nv_bfloat16>(uint32_t most, uint32_t x)
{
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<__nv_bfloat162 *>(&most), __habs2(*reinterpret_cast<__nv_bfloat162 *>(&x)));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// The word with 0 in their place.
template <typename T> __device__ __forceinline__ uint32_t wf_fit(uint32_t x)
{
    constexpr int kBits = 8 * sizeof(T);
    return x & ~((wf_unfit<T>(x) >> (kBits - 1)) * ((1u << kBits) - 1));
}
template <typename T> __device__ __forceinline__ uint4 wf_fit(const uint4 &x)
{
    return make_uint4(wf_fit<T>(x.x), wf_fit<T>(x.y), wf_fit<T>(x.z), wf_fit<T>(x.w));
}

// Rounded to nearest, even; beyond 448 to +-448; a in the lower byte.
__device__ __forceinline__ uint32_t wf_e4m3_of(float a, float b)
{
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
