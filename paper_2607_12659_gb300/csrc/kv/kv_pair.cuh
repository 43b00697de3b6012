// Two fp32 numbers by one instruction.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace jpi {
namespace {

__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
    uint64_t r, a = *reinterpret_cast<uint64_t*>(&x), b = *reinterpret_cast<uint64_t*>(&y);
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
    uint64_t r, a = *reinterpret_cast<uint64_t*>(&x), b = *reinterpret_cast<uint64_t*>(&y), c = *reinterpret_cast<uint64_t*>(&z);
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return *reinterpret_cast<float2*>(&r);
}

}  // namespace
}  // namespace jpi
