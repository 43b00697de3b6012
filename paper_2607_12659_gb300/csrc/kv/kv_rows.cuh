// What the row kernels of attend and weigh share (kv_attend.cu, kv_weigh.cu): the rows of a side, loads of
// keys and values straight into the fragments of mma.sync, and the small pieces around them.
//
// Rows. The query tokens and heads that read the same keys form one matrix: for a prefix the n tokens of the
// run's requests x the gq query heads of a KV head, for a request's own rows its tokens x gq. Row r is
// query token r / gq of the run (or request), head kvh * gq + r % gq. A warp takes 8 of them.
//
// Keys are the 16 rows of an mma.sync m16n8k16 and query rows its 8 columns, so that 8 query rows (one token of
// eight heads) waste nothing.

#pragma once

#include "kv.h"
#include "../ptx.h"

namespace jpi {
namespace {

constexpr int KR_ROWS = 8;    // query rows of a warp

// Where a warp's query rows live.
struct RowTile {
    long long tok0;   // first query token of the run or request, in batch * tokens order
    int head0;        // kvh * gq
    int r0, R;        // first row of the tile, rows in all
};

__device__ __forceinline__ long long row_token(const KvCall& c, const RowTile& t, int r) { return t.tok0 + c.by_gq.div((uint32_t)r); }
// Its index in [batch][tokens][H], and its first element in q.
__device__ __forceinline__ long long row_index(const KvCall& c, const RowTile& t, int r) {
    uint32_t h;
    const uint32_t tok = c.by_gq.div((uint32_t)r, h);
    return (t.tok0 + tok) * c.H + t.head0 + h;
}
__device__ __forceinline__ long long row_query(const KvCall& c, const RowTile& t, int r) {
    uint32_t h;
    const uint32_t tok = c.by_gq.div((uint32_t)r, h);
    return (t.tok0 + tok) * c.q_stride + (long long)(t.head0 + h) * c.D;
}
// Keys that row r sees on its side.
__device__ __forceinline__ int row_seen(const KvCall& c, bool prefix, int cache, const RowTile& t, int r) {
    if (r >= t.R) return 0;
    const KvSide& s = prefix ? c.prefix : c.own;
    const int n = prefix ? s.len[cache] : s.len[row_token(c, t, r)];
    return min(max(n, 0), s.rows);
}

constexpr float KR_LOG2E = 1.4426950408889634f;
// 2^x by the hardware approximation (PTX ex2.approx.ftz.f32, relative error ~2^-22).
__device__ __forceinline__ float kr_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// D += A B, A 16 x 16 (row), B 16 x 8 (col), bf16 operands, fp32 sums.
__device__ __forceinline__ void kr_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Transposes an 8 x 8 matrix of 16-bit elements spread over the warp.
__device__ __forceinline__ uint32_t kr_transpose(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t kr_pack(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint4 kr_ld(const void* p, bool ok) {
    return ok ? __ldg(static_cast<const uint4*>(p)) : make_uint4(0, 0, 0, 0);
}

}  // namespace
}  // namespace jpi
