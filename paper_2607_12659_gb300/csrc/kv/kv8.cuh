// A cache held in 8 bits: e4m3 codes and the bytes of their scales (kv8_append.cu, kv_span.cu, kv_span_t5.cu).
#pragma once

#include "kv.h"

#include <cuda_fp16.h>

#include <algorithm>

namespace jpi {
namespace {

// 2^(e - 127): 0 from e = 0 down (the numbers below 2^-126 are not used).
__device__ __forceinline__ float kv8_pow2(int e) { return __int_as_float(max(e, 0) << 23); }

// What a scale's byte stands for.
__device__ __forceinline__ float kv8_scale(uint32_t s) {
    return __uint_as_float(s == 255 ? 0x7fffffffu : s == 0 ? 0x00400000u : s << 23);
}

// The byte of the least scale at which `top` (finite, >= 0) is at most 448 = 1.75 2^8.
__device__ __forceinline__ int kv8_exponent(float top) {
    const uint32_t b = __float_as_uint(top);
    return max((int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u), 1);
}

// Four codes, the first lowest; infinities and NaN are held as NaN.
__device__ __forceinline__ uint32_t kv8_codes(float x0, float x1, float x2, float x3) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x1), "f"(x0));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x3), "f"(x2));
    uint32_t r = (uint32_t)lo | (uint32_t)hi << 16;
    if (fabsf(x0) == INFINITY) r |= 0x7fu;
    if (fabsf(x1) == INFINITY) r |= 0x7f00u;
    if (fabsf(x2) == INFINITY) r |= 0x7f0000u;
    if (fabsf(x3) == INFINITY) r |= 0x7f000000u;
    return r;
}

// Two codes (the low one first) as fp16 numbers: e4m3 is a subset of them, NaN included.
__device__ __forceinline__ uint32_t kv8_half2(uint32_t codes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
    return r;
}
__device__ __forceinline__ void kv8_values(uint32_t codes, float (&z)[4]) {
    const uint32_t lo = kv8_half2(codes & 0xffffu), hi = kv8_half2(codes >> 16);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    z[0] = a.x;
    z[1] = a.y;
    z[2] = b.x;
    z[3] = b.y;
}

}  // namespace
}  // namespace jpi
