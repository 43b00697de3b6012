// What the kernels that code heads share (kv_append.cu, kv_append_normed.cu, kv8_append.cu): rotary modes, 16-byte pieces of a
// head, and a pair's angle.
#pragma once

#include "kv.h"

namespace jpi {
namespace {

enum RopeMode {
    RM_NONE = 0,     // copy
    RM_HALF = 1,     // pairs (d, d + dim / 2), whole chunks of both
    RM_INTER = 2,    // pairs (2 i, 2 i + 1), within a chunk
    RM_SCALAR = 3    // the half layout where dim / 2 is no whole number of chunks: element by element
};

template <typename E>
struct Chunk {   // 16 bytes of E as fp32
    static constexpr int V = 16 / sizeof(E);
    __device__ static __forceinline__ void unpack(uint4 u, float (&x)[V]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 2) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            } else {
                x[i] = __uint_as_float(w[i]);
            }
        }
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[V]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 2) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&b);
            } else {
                w[i] = __float_as_uint(x[i]);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// (cos, sin) of `position` times the pair's turns, times m.
__device__ __forceinline__ float2 phase(int position, uint64_t turns, float m) {
    const uint64_t ph = (uint64_t)(int64_t)position * turns;
    float s, c;
    sincospif((float)(int32_t)(ph >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns in [-1, 1)
    return make_float2(c * m, s * m);
}

// The same with the angle reduced to an eighth of a turn before it becomes an fp32 number: off by 2^-28 turns in place of 2^-26, for
// codes of 8 bits, where each value beside a border that falls to the other side is a step of its own. On |x| <= 1/4 half turns the
// series of sin(pi x) and cos(pi x) to x^9 and x^10 leave 2^-29 and 2^-33, in a third of sincospif's instructions.
__device__ __forceinline__ float2 phase_near(int position, uint64_t turns, float m) {
    const uint64_t ph = (uint64_t)(int64_t)position * turns;
    const uint32_t hi = (uint32_t)(ph >> 32), quarter = (hi + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(hi - (quarter << 30)) * 4.656612873077393e-10f, z = x * x;
    const float s = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 0.0821458866f, -0.599264529f), 2.55016404f), -5.16771278f), 3.14159265f);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -0.0258068914f, 0.23533063f), -1.33526277f), 4.05871213f), -4.9348022f), 1.f);
    const float u = quarter & 1 ? s : c, v = quarter & 1 ? c : s;
    // (c, s), (-s, c), (-c, -s), (s, -c)
    return make_float2((quarter + 1) & 2 ? -u * m : u * m, quarter & 2 ? -v * m : v * m);
}

constexpr int AP_MAX_PAIRS = 128;   // dim / 2

}  // namespace
}  // namespace jpi
