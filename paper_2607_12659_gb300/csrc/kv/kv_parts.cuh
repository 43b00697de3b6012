// The parts of an attention call (kv_attend.cu, kv_span.cu): how a side is dealt to blocks, the partial rows that these
// leave in the workspace, and how the warps of a block join theirs.
#pragma once

#include "kv_rows.cuh"

namespace jpi {
namespace {

constexpr int AT_WARPS = 4;
constexpr int AT_THREADS = 32 * AT_WARPS;

// How one side is dealt to blocks: `wr` warps of a block take different row tiles, and each of those `wk` warps
// different keys.
struct SidePlan {
    int wr = 1, wk = 1;
    int tiles = 0;        // blocks of wr row tiles per cache and KV head
    int splits = 0;       // key ranges
    long long blocks = 0;
    KvDiv by_splits, by_tiles;
};

struct AttendArgs {
    KvCall c;
    SidePlan p, o;
    float* po;            // [parts][rows][D] unnormalised outputs
    float2* pml;          // [rows][parts] (m, l), m unscaled
    int parts;
    float c2;             // log2(e) * scale
    long long rows;       // batch * tokens * H
    void* out;            // rows of one part: the result itself, else null
    float* lse;
};

// The block's piece of work: side, cache, KV head, row tile and key split.
struct Piece {
    bool prefix;
    int cache, kvh, part;
    uint32_t split;
    RowTile t;
};
__device__ __forceinline__ Piece piece_of(const AttendArgs& a, long long piece, int warp) {
    Piece x;
    uint32_t i = (uint32_t)piece, tile, kvh;
    x.prefix = i < a.p.blocks;
    if (!x.prefix) i -= (uint32_t)a.p.blocks;
    const SidePlan& s = x.prefix ? a.p : a.o;
    i = s.by_splits.div(i, x.split);
    i = s.by_tiles.div(i, tile);
    x.cache = (int)a.c.by_K.div(i, kvh);
    x.part = (x.prefix ? 0 : a.p.splits) + (int)x.split;
    const int toks = x.prefix ? a.c.batch / a.c.groups * a.c.tokens : a.c.tokens;
    x.t.tok0 = (long long)x.cache * toks;
    x.kvh = (int)kvh;
    x.t.head0 = (int)kvh * a.c.gq;
    x.t.R = toks * a.c.gq;
    x.t.r0 = ((int)tile * s.wr + warp / s.wk) * KR_ROWS;
    return x;
}

// Shared memory of one warp's share of the merge: 8 rows of DP outputs, then (m, l) per row. BYTES: of a block of
// AT_WARPS warps, which holds the query fragments in it before.
template <int DP>
struct MergeSmem {
    static constexpr int LD = DP + 4;   // the row pad spreads the rows over the banks
    static constexpr int WARP_FLOATS = KR_ROWS * LD + 2 * KR_ROWS;
    static constexpr int BYTES = AT_WARPS * WARP_FLOATS * 4;
};

// One row's elements as a warp holds them: lane's float4 i is d = 4 lane + 128 i.
template <int DP>
struct RowAcc {
    static constexpr int NI = (DP + 127) / 128;
    float4 o[NI];
    float m, l;
    __device__ __forceinline__ void add(float w, const float4 (&v)[NI]) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            o[i].x = fmaf(w, v[i].x, o[i].x);
            o[i].y = fmaf(w, v[i].y, o[i].y);
            o[i].z = fmaf(w, v[i].z, o[i].z);
            o[i].w = fmaf(w, v[i].w, o[i].w);
        }
    }
};

// What a row's outputs are multiplied by: 0 without a key, NaN with a NaN score.
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float log_sum(float m, float l, float scale) { return l == 0.f ? -INFINITY : fmaf(m, scale, logf(l)); }

// The row's result from its joined sums, elements from d0 on.
template <int DP, typename E>
__device__ __forceinline__ void write_row(const AttendArgs& a, const RowAcc<DP>& r, long long row, int d0, int lane) {
    const float inv = inverse_sum(r.l);
    E* out = static_cast<E*>(a.out) + row * a.c.D;
#pragma unroll
    for (int i = 0; i < RowAcc<DP>::NI; ++i) {
        const int d = d0 + 4 * lane + 128 * i;
        if (d >= a.c.D) continue;
        const float4 v = make_float4(r.o[i].x * inv, r.o[i].y * inv, r.o[i].z * inv, r.o[i].w * inv);
        if constexpr (sizeof(E) == 2)
            *(uint2*)(out + d) = make_uint2(kr_pack(v.x, v.y), kr_pack(v.z, v.w));
        else
            *(float4*)(out + d) = v;
    }
    if (d0 == 0 && lane == 0 && a.lse) a.lse[row] = log_sum(r.m, r.l, a.c.scale);
}

// Joins the key warps of each row tile (their outputs and (m, l) are in shared memory) and writes the part, or, where
// the block's keys are the last of its rows, the result.
template <int DP, typename E>
__device__ __forceinline__ void merge_and_write(const AttendArgs& a, const Piece& x, const SidePlan& s, const float* sm, int warp,
                                                int lane) {
    using M = MergeSmem<DP>;
    constexpr int NI = RowAcc<DP>::NI;
    __syncthreads();
    // Every warp takes rows (its index among the key warps) + n wk of its row tile.
    const float* tile = sm + (warp / s.wk) * s.wk * M::WARP_FLOATS;
    for (int rr = warp % s.wk; rr < KR_ROWS; rr += s.wk) {
        const int r = x.t.r0 + rr;
        if (r >= x.t.R) continue;
        const long long row = row_index(a.c, x.t, r);
        RowAcc<DP> acc;
        acc.m = -INFINITY;
        acc.l = 0.f;
        for (int k = 0; k < s.wk; ++k) acc.m = fmaxf(acc.m, tile[k * M::WARP_FLOATS + KR_ROWS * M::LD + 2 * rr]);
#pragma unroll
        for (int i = 0; i < NI; ++i) acc.o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < s.wk; ++k) {
            const float* f = tile + k * M::WARP_FLOATS;
            const float mk = f[KR_ROWS * M::LD + 2 * rr], lk = f[KR_ROWS * M::LD + 2 * rr + 1];
            if (lk == 0.f) continue;
            const float w = mk == -INFINITY ? 0.f : kr_ex2((mk - acc.m) * a.c2);
            acc.l += w * lk;
            float4 v[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int d = 4 * lane + 128 * i;
                v[i] = d < DP ? *(const float4*)(f + rr * M::LD + d) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            acc.add(w, v);
        }
        if (a.out) {
            write_row<DP, E>(a, acc, row, 0, lane);
            continue;
        }
        const long long at = x.part * a.rows + row;
        if (lane == 0) a.pml[row * a.parts + x.part] = make_float2(acc.m, acc.l);
        if (acc.l != 0.f) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int d = 4 * lane + 128 * i;
                if (d < a.c.D) *(float4*)(a.po + at * a.c.D + d) = acc.o[i];
            }
        }
    }
}

// Rows of partial outputs the workspace holds.
inline long long ws_rows(const jpi_kv_handle* h) {
    const long long rows = (long long)h->cfg.max_batch * h->cfg.max_tokens * h->H;
    return 2 * rows + 512ll * h->num_sms;
}

}  // namespace
}  // namespace jpi
