// What the kernels of 128-row tiles share (kv_attend_t5.cu, kv_span_t5.cu).
#pragma once

#include "kv_rows.cuh"

namespace jpi {
namespace {

// (a - m) c for two scores at a time.
__device__ __forceinline__ void sub_scale2(float a, float b, uint64_t neg_m2, uint64_t c2, float& x, float& y) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(neg_m2));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(c2));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
}
// a c - m likewise, the products rounded: 0 for the a that m is the product of. (The sums one at a time: the assembler makes one
// instruction of a product and a sum of pairs, with one rounding, .rn or not.)
__device__ __forceinline__ void scale_sub2(float a, float b, uint64_t c2, float m, float& x, float& y) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(c2));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
    x = __fsub_rn(x, m);
    y = __fsub_rn(y, m);
}
__device__ __forceinline__ uint64_t pair2(float a) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %1};" : "=l"(v) : "f"(a));
    return v;
}

// Whether any of the `n` threads that share named barrier `id` says so.
__device__ __forceinline__ bool group_any(uint32_t id, uint32_t n, bool mine) {
    uint32_t r;
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.u32 p, %3, 0;\n bar.red.or.pred q, %1, %2, p;\n selp.u32 %0, 1, 0, q;\n}"
        : "=r"(r)
        : "r"(id), "r"(n), "r"((uint32_t)mine)
        : "memory");
    return r != 0;
}

// Whether one of two bf16 values is an infinity or NaN.
__device__ __forceinline__ bool bad_pair(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }

}  // namespace
}  // namespace jpi
