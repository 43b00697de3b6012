// Attention of a batch over shared prefixes and own rows (jpi_kv_attend).
//
//   o_r = sum_j p_rj v_j,  p_rj = exp(s_rj - lse_r),  s_rj = scale q_r . k_j,
// j over the first prefix_len rows of the run's prefix and then the first `seen` rows of the request's own
// cache. A prefix is read once for all its requests: their query rows are one matrix.
//
// The softmax is computed in parts: every part (a range of keys of one side) keeps a running maximum m and
// sum l per row and an unnormalised output, all fp32, and they are joined as
//   o = sum_s w_s O_s / sum_s w_s l_s,  w_s = exp(scale (m_s - M)),
// in part order, so that a result does not depend on which block finished first. A part that saw no key
// has m = -inf and weighs nothing; a row of only such parts is zero. Maxima are those of the unscaled
// products, and the difference is scaled, not the product: log2(e) times a score near the type's largest
// values would overflow.
//
// Kernels: the row kernels here take both sides, 8 query rows a warp; many rows on one prefix (from 32) go to
// tiles of 128 rows instead (kv_attend_t5.cu), bound by tensor cores and 2^x where the row kernel is bound by
// memory, so the two share the SMs: the row kernel starts first with two blocks per SM, the tiles start while it
// runs. k_kv_combine joins the parts, except where a row has only one.

#include "kv_rows.cuh"
#include "kv_attend.h"
#include "kv_maps.h"

#include <algorithm>

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
};

struct AttendArgs {
    KvCall c;
    SidePlan p, o;
    float* po;            // [parts][rows][D] unnormalised outputs
    float2* pml;          // [parts][rows] (m, l), m unscaled
    float c2;             // log2(e) * scale
    long long rows;       // batch * tokens * H
    void* out;            // rows of one part: the result itself, else null
    float* lse;
    int* err;
};

// The block's piece of work: side, cache, KV head, row tile and key split.
struct Piece {
    bool prefix;
    int cache, split, part;
    RowTile t;
    int wk, nwk;
};
__device__ __forceinline__ Piece piece_of(const AttendArgs& a, long long piece, int warp) {
    Piece x;
    uint32_t i = (uint32_t)piece;
    x.prefix = i < a.p.blocks;
    if (!x.prefix) i -= (uint32_t)a.p.blocks;
    const SidePlan& s = x.prefix ? a.p : a.o;
    x.split = (int)(i % (uint32_t)s.splits);
    i /= (uint32_t)s.splits;
    const int tile = (int)(i % (uint32_t)s.tiles);
    i /= (uint32_t)s.tiles;
    const int kvh = (int)(i % (uint32_t)a.c.K);
    x.cache = (int)(i / (uint32_t)a.c.K);
    x.part = x.prefix ? x.split : a.p.splits + x.split;
    const int toks = x.prefix ? a.c.batch / a.c.groups * a.c.tokens : a.c.tokens;
    x.t.tok0 = (long long)x.cache * toks;
    x.t.head0 = kvh * a.c.gq;
    x.t.R = toks * a.c.gq;
    x.t.r0 = (tile * s.wr + warp / s.wk) * KR_ROWS;
    x.wk = warp % s.wk;
    x.nwk = s.wk;
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

// Joins parts first, first + step, .. of a row's `parts` to what `r` holds, all relative to the largest maximum
// of the row (which r.m becomes). The loads of JOIN parts are in flight together: they are made whether the part
// weighs anything or not (its memory is the workspace's), and a part of no weight, which may never have been
// written, is replaced by zeros.
template <int DP>
__device__ __forceinline__ void join_parts(const AttendArgs& a, RowAcc<DP>& r, long long row, int parts, int first, int step,
                                           int lane) {
    constexpr int NI = RowAcc<DP>::NI, JOIN = 16 / NI;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < parts) ml = __ldcg(&a.pml[lane * a.rows + row]);
    float M = fmaxf(r.m, ml.x);
    for (int p = 32 + lane; p < parts; p += 32) M = fmaxf(M, __ldcg(&a.pml[p * a.rows + row]).x);
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, e));
    const float w0 = r.m == -INFINITY ? 0.f : kr_ex2((r.m - M) * a.c2);
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) r.o[i] = make_float4(r.o[i].x * w0, r.o[i].y * w0, r.o[i].z * w0, r.o[i].w * w0);
    int d[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) d[i] = 4 * lane + 128 * i < a.c.D ? 4 * lane + 128 * i : 0;
    for (int p0 = 0; p0 < parts; p0 += 32) {
        if (p0 > 0) {
            ml = make_float2(-INFINITY, 0.f);
            if (p0 + lane < parts) ml = __ldcg(&a.pml[(p0 + lane) * a.rows + row]);
        }
        const float w = ml.x == -INFINITY ? 0.f : kr_ex2((ml.x - M) * a.c2);
        if ((p0 + lane) % step == first) l += w * ml.y;   // (w = 0 past the parts)
        const int n = min(32, parts - p0);
        for (int k0 = first; k0 < n; k0 += JOIN * step) {   // step divides 32
            float4 v[JOIN][NI];
            float wk[JOIN];
#pragma unroll
            for (int k = 0; k < JOIN; ++k) {
                const int q = min(k0 + k * step, n - 1);
                const float* src = a.po + ((p0 + q) * a.rows + row) * a.c.D;
                wk[k] = __shfl_sync(0xffffffffu, w, q);
                if (k0 + k * step >= n) wk[k] = 0.f;
#pragma unroll
                for (int i = 0; i < NI; ++i) v[k][i] = __ldcg((const float4*)(src + d[i]));
            }
#pragma unroll
            for (int k = 0; k < JOIN; ++k) {
#pragma unroll
                for (int i = 0; i < NI; ++i)
                    if (wk[k] == 0.f) v[k][i] = make_float4(0.f, 0.f, 0.f, 0.f);
                r.add(wk[k], v[k]);
            }
        }
    }
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) l += __shfl_xor_sync(0xffffffffu, l, e);
    r.l = r.l * w0 + l;
    r.m = M;
}

// The row's result from its joined sums.
template <int DP, typename E>
__device__ __forceinline__ void write_row(const AttendArgs& a, const RowAcc<DP>& r, long long row, int lane) {
    const float inv = r.l > 0.f ? 1.f / r.l : 0.f;   // (a NaN sum comes with NaN outputs)
    E* out = static_cast<E*>(a.out) + row * a.c.D;
#pragma unroll
    for (int i = 0; i < RowAcc<DP>::NI; ++i) {
        const int d = 4 * lane + 128 * i;
        if (d >= a.c.D) continue;
        const float4 v = make_float4(r.o[i].x * inv, r.o[i].y * inv, r.o[i].z * inv, r.o[i].w * inv);
        if constexpr (sizeof(E) == 2)
            *(uint2*)(out + d) = make_uint2(kr_pack(v.x, v.y), kr_pack(v.z, v.w));
        else
            *(float4*)(out + d) = v;
    }
    if (lane == 0 && a.lse) a.lse[row] = r.m == -INFINITY ? -INFINITY : fmaf(r.m, a.c.scale, logf(r.l));
}

// Joins the key warps of each row tile (their outputs and (m, l) are in shared memory) and writes the part, or, where
// the block's keys are the last of its rows, the result.
template <int DP, typename E>
__device__ __forceinline__ void merge_and_write(const AttendArgs& a, const Piece& x, const SidePlan& s, const float* sm, int warp,
                                                int lane) {
    using M = MergeSmem<DP>;
    constexpr int NI = RowAcc<DP>::NI;
    __syncthreads();
    // Every warp takes rows (its index among the key warps) + n nwk of its row tile.
    const float* tile = sm + (warp / s.wk) * s.wk * M::WARP_FLOATS;
    for (int rr = x.wk; rr < KR_ROWS; rr += x.nwk) {
        const int r = x.t.r0 + rr;
        if (r >= x.t.R) continue;
        const long long row = row_index(x.t, a.c.gq, a.c.H, r);
        RowAcc<DP> acc;
        acc.m = -INFINITY;
        acc.l = 0.f;
        for (int k = 0; k < x.nwk; ++k) acc.m = fmaxf(acc.m, tile[k * M::WARP_FLOATS + KR_ROWS * M::LD + 2 * rr]);
#pragma unroll
        for (int i = 0; i < NI; ++i) acc.o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < x.nwk; ++k) {
            const float* f = tile + k * M::WARP_FLOATS;
            const float mk = f[KR_ROWS * M::LD + 2 * rr];
            if (mk == -INFINITY) continue;
            const float w = kr_ex2((mk - acc.m) * a.c2);
            acc.l += w * f[KR_ROWS * M::LD + 2 * rr + 1];
            float4 v[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int d = 4 * lane + 128 * i;
                v[i] = d < DP ? *(const float4*)(f + rr * M::LD + d) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            acc.add(w, v);
        }
        if (a.out) {
            write_row<DP, E>(a, acc, row, lane);
            continue;
        }
        const long long at = x.part * a.rows + row;
        if (lane == 0) a.pml[at] = make_float2(acc.m, acc.l);
        if (acc.m != -INFINITY) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int d = 4 * lane + 128 * i;
                if (d < a.c.D) *(float4*)(a.po + at * a.c.D + d) = acc.o[i];
            }
        }
    }
}

// bf16, any head dim to DP: one warp = 8 query rows over the 16-key blocks wk, wk + nwk, .. of the split.
// Probabilities enter the second product as two bf16 terms (the rounded value and what the rounding left), so
// that its error stays that of fp32 sums: the products are bound by the loads of keys and values, and the
// second term costs no time there.
template <int DP>
__global__ void __launch_bounds__(AT_THREADS, 2) k_kv_attend_mma(const __grid_constant__ AttendArgs a) {
    extern __shared__ __align__(16) float kv_smem[];
    constexpr int NC = DP / 32;    // chunk groups of a key
    constexpr int NV = DP / 64;    // chunk groups of a value row
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, j = lane & 3;
    ptx::grid_dep_launch();
    const Piece x = piece_of(a, blockIdx.x, warp);
    const SidePlan& sp = x.prefix ? a.p : a.o;
    const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
    const int D = a.c.D;
    uint4* qs = reinterpret_cast<uint4*>(kv_smem) + (warp / sp.wk) * (NC * 32);
    if (x.wk == 0) load_q_frags<DP>(a.c, x.t, qs, lane);
    // Keys this lane's two rows (columns 2 j, 2 j + 1 of the products) see, and the most any row of the tile sees.
    const int n0 = row_seen(a.c, x.prefix, x.cache, x.t, x.t.r0 + 2 * j);
    const int n1 = row_seen(a.c, x.prefix, x.cache, x.t, x.t.r0 + 2 * j + 1);
    int lim = max(n0, n1), low = 0x7fffffff;
    if (x.t.r0 + 2 * j < x.t.R) low = n0;
    if (x.t.r0 + 2 * j + 1 < x.t.R) low = min(low, n1);
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lim = max(lim, __shfl_xor_sync(0xffffffffu, lim, o));
        low = min(low, __shfl_xor_sync(0xffffffffu, low, o));
    }
    __syncthreads();
    const long long nb = (lim + KR_KEYS - 1) / KR_KEYS;
    const int b0 = (int)(nb * x.split / sp.splits), b1 = (int)(nb * (x.split + 1) / sp.splits);
    const __nv_bfloat16* kbase = (const __nv_bfloat16*)s.k + x.cache * s.cs + (x.t.head0 / a.c.gq) * s.hs;
    const __nv_bfloat16* vbase = (const __nv_bfloat16*)s.v + x.cache * s.cs + (x.t.head0 / a.c.gq) * s.hs;
    float o[NV][4][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][t][e] = 0.f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
    for (int blk = b0 + x.wk; blk < b1; blk += x.nwk) {
        const int key0 = blk * KR_KEYS;
        uint4 kf[NC][2], vf[NV][4];
        {
            const __nv_bfloat16* kp = kbase + (long long)(key0 + g) * s.rs + 8 * j;
            const bool ok0 = key0 + g < lim, ok1 = key0 + g + 8 < lim;
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const bool in = 8 * (4 * i + j) < D;
                kf[i][0] = kr_ld(kp + 32 * i, ok0 && in);
                kf[i][1] = kr_ld(kp + 8 * s.rs + 32 * i, ok1 && in);
            }
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int key = key0 + 2 * j + (h & 1) + 8 * (h >> 1);
            const __nv_bfloat16* vp = vbase + (long long)key * s.rs + 8 * g;
#pragma unroll
            for (int i = 0; i < NV; ++i) vf[i][h] = kr_ld(vp + 64 * i, key < lim && 8 * (g + 8 * i) < D);
        }
        float sc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const uint4 q = qs[32 * i + lane];
            kr_mma(sc, kf[i][0].x, kf[i][1].x, kf[i][0].y, kf[i][1].y, q.x, q.y);
            kr_mma(sc, kf[i][0].z, kf[i][1].z, kf[i][0].w, kf[i][1].w, q.z, q.w);
        }
        // Scores of keys g, g + 8 and rows 2 j, 2 j + 1; hidden ones are replaced, whatever they hold.
        const float s00 = key0 + g < n0 ? sc[0] : -INFINITY;
        const float s01 = key0 + g < n1 ? sc[1] : -INFINITY;
        const float s10 = key0 + g + 8 < n0 ? sc[2] : -INFINITY;
        const float s11 = key0 + g + 8 < n1 ? sc[3] : -INFINITY;
        float x0 = fmaxf(s00, s10), x1 = fmaxf(s01, s11);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, d));
            x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, d));
        }
        if (__any_sync(0xffffffffu, x0 > m0 || x1 > m1)) {
            const float y0 = fmaxf(m0, x0), y1 = fmaxf(m1, x1);
            const float a0 = m0 == -INFINITY ? 0.f : kr_ex2((m0 - y0) * a.c2), a1 = m1 == -INFINITY ? 0.f : kr_ex2((m1 - y1) * a.c2);
            m0 = y0;
            m1 = y1;
            l0 *= a0;
            l1 *= a1;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    o[i][t][0] *= a0;
                    o[i][t][1] *= a1;
                    o[i][t][2] *= a0;
                    o[i][t][3] *= a1;
                }
        }
        const float f0 = m0 == -INFINITY ? 0.f : m0, f1 = m1 == -INFINITY ? 0.f : m1;
        const float p00 = kr_ex2((s00 - f0) * a.c2), p01 = kr_ex2((s01 - f1) * a.c2);
        const float p10 = kr_ex2((s10 - f0) * a.c2), p11 = kr_ex2((s11 - f1) * a.c2);
        l0 += p00 + p10;
        l1 += p01 + p11;
        const uint32_t h0 = kr_pack(p00, p01), h1 = kr_pack(p10, p11);
        const uint32_t e0 = kr_pack(p00 - __uint_as_float(h0 << 16), p01 - __uint_as_float(h0 & 0xffff0000u));
        const uint32_t e1 = kr_pack(p10 - __uint_as_float(h1 << 16), p11 - __uint_as_float(h1 & 0xffff0000u));
        const uint32_t ph0 = kr_transpose(h0), ph1 = kr_transpose(h1), pe0 = kr_transpose(e0), pe1 = kr_transpose(e1);
        auto product = [&](uint32_t bh0, uint32_t bh1, uint32_t be0, uint32_t be1) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t v0[4] = {vf[i][0].x, vf[i][0].y, vf[i][0].z, vf[i][0].w};
                const uint32_t v1[4] = {vf[i][1].x, vf[i][1].y, vf[i][1].z, vf[i][1].w};
                const uint32_t v2[4] = {vf[i][2].x, vf[i][2].y, vf[i][2].z, vf[i][2].w};
                const uint32_t v3[4] = {vf[i][3].x, vf[i][3].y, vf[i][3].z, vf[i][3].w};
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const uint32_t a0 = __byte_perm(v0[t], v1[t], 0x5410), a1 = __byte_perm(v0[t], v1[t], 0x7632);
                    const uint32_t a2 = __byte_perm(v2[t], v3[t], 0x5410), a3 = __byte_perm(v2[t], v3[t], 0x7632);
                    kr_mma(o[i][t], a0, a1, a2, a3, bh0, bh1);
                    kr_mma(o[i][t], a0, a1, a2, a3, be0, be1);
                }
            }
        };
        // A block that some rows see only a part of: 0 times an infinity or NaN that one row sees and another does
        // not would reach the other. Where it holds such a value, row by row over the row's own keys.
        bool odd = false;
        if (low < min(key0 + KR_KEYS, lim)) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const uint32_t v[4] = {vf[i][h].x, vf[i][h].y, vf[i][h].z, vf[i][h].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        odd = odd || (v[e] & 0x7f80u) == 0x7f80u || (v[e] & 0x7f800000u) == 0x7f800000u;
                }
            odd = __any_sync(0xffffffffu, odd);
        }
        if (!odd) {
            product(ph0, ph1, pe0, pe1);
        } else {
            for (int r = KR_ROWS - 1; r >= 0; --r) {
                // Row r's count, from a lane that holds it.
                const int nr = __shfl_sync(0xffffffffu, (r & 1) ? n1 : n0, r >> 1);
                uint4 keep_v[NV][4];
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        keep_v[i][h] = vf[i][h];
                        if (key0 + 2 * j + (h & 1) + 8 * (h >> 1) >= nr) vf[i][h] = make_uint4(0, 0, 0, 0);
                    }
                const bool mine = g == r;
                product(mine ? ph0 : 0u, mine ? ph1 : 0u, mine ? pe0 : 0u, mine ? pe1 : 0u);
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int h = 0; h < 4; ++h) vf[i][h] = keep_v[i][h];
            }
        }
    }
    // Sums over the key lanes.
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, d);
        l1 += __shfl_xor_sync(0xffffffffu, l1, d);
    }
    __syncthreads();   // the query fragments have been read
    float* f = kv_smem + warp * MergeSmem<DP>::WARP_FLOATS;
    constexpr int LD = MergeSmem<DP>::LD;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int d = 8 * (g + 8 * i);
        *(float4*)(f + (2 * j) * LD + d) = make_float4(o[i][0][0], o[i][0][2], o[i][1][0], o[i][1][2]);
        *(float4*)(f + (2 * j) * LD + d + 4) = make_float4(o[i][2][0], o[i][2][2], o[i][3][0], o[i][3][2]);
        *(float4*)(f + (2 * j + 1) * LD + d) = make_float4(o[i][0][1], o[i][0][3], o[i][1][1], o[i][1][3]);
        *(float4*)(f + (2 * j + 1) * LD + d + 4) = make_float4(o[i][2][1], o[i][2][3], o[i][3][1], o[i][3][3]);
    }
    if (g == 0) {
        float* ml = f + KR_ROWS * LD + 4 * j;
        ml[0] = m0;
        ml[1] = l0;
        ml[2] = m1;
        ml[3] = l1;
    }
    merge_and_write<DP, __nv_bfloat16>(a, x, sp, kv_smem, warp, lane);
}

// The same work for caches that bulk tensor copies can read (head dims from 64, see kv_maps.h): each warp
// streams its 16 KB blocks of 16 (D = 256) to 64 (D = 64) keys through shared memory of its own, the next keys on
// their way while this block's values are used and the other way round, and reads fragments with ldmatrix. Against loads
// to registers this needs half the registers and no room in L1 for what is in flight, so that a block fits beside
// the 128-row tiles on their SM. Blocks are persistent: piece blockIdx.x, + gridDim.x, ..
constexpr int RT_WARPS = 2;
constexpr int RT_THREADS = 32 * RT_WARPS;
constexpr int RT_BLOCK = 16384;   // bytes of a warp's keys and values
constexpr uint64_t RT_WAIT_NS = 200ull * 1000 * 1000;

template <int DP>
struct RtSmem {
    static constexpr int KEYS = RT_BLOCK / (4 * DP);   // keys of a block
    static constexpr int HALF = RT_BLOCK / 2;          // its keys, then its values
    static constexpr int BAR_OFF = RT_WARPS * RT_BLOCK > RT_WARPS * MergeSmem<DP>::WARP_FLOATS * 4
                                       ? RT_WARPS * RT_BLOCK
                                       : RT_WARPS * MergeSmem<DP>::WARP_FLOATS * 4;
    static constexpr int BYTES = BAR_OFF + 8 * 2 * RT_WARPS;
};

struct RtMaps {
    CUtensorMap k[2], v[2];   // prefix, own
    int3 at[2];
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}

template <int DP>
__global__ void __launch_bounds__(RT_THREADS) k_kv_attend_rows(const __grid_constant__ RtMaps maps,
                                                               const __grid_constant__ AttendArgs a) {
    using L = RtSmem<DP>;
    extern __shared__ __align__(1024) uint8_t rt_smem[];
    constexpr int MT = L::KEYS / 16;   // 16-key tiles of a block
    constexpr int ND = DP / 16;
    const int warp = ptx::warp_index(), lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
    uint8_t* block = rt_smem + warp * RT_BLOCK;
    const uint32_t ks = ptx::smem_u32(block), vs = ks + L::HALF;
    uint64_t* bar = (uint64_t*)(rt_smem + L::BAR_OFF) + 2 * warp;   // keys, values
    ptx::grid_dep_launch();
    if (lane == 0) {
        ptx::mbar_init(&bar[0], 1);
        ptx::mbar_init(&bar[1], 1);
        ptx::fence_mbar_init();
    }
    __syncwarp();
    int asked[2] = {0, 0}, done[2] = {0, 0};   // copies asked for and waited for, of keys and of values
    bool good = true;
    const long long pieces = a.p.blocks + a.o.blocks;
    for (long long piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        const Piece x = piece_of(a, piece, warp);
        const SidePlan& sp = x.prefix ? a.p : a.o;
        const int side = x.prefix ? 0 : 1;
        const int kvh = x.t.head0 / a.c.gq;
        const int n0 = row_seen(a.c, x.prefix, x.cache, x.t, x.t.r0 + 2 * j);
        const int n1 = row_seen(a.c, x.prefix, x.cache, x.t, x.t.r0 + 2 * j + 1);
        int lim = max(n0, n1), low = 0x7fffffff;
        if (x.t.r0 + 2 * j < x.t.R) low = n0;
        if (x.t.r0 + 2 * j + 1 < x.t.R) low = min(low, n1);
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            lim = max(lim, __shfl_xor_sync(0xffffffffu, lim, o));
            low = min(low, __shfl_xor_sync(0xffffffffu, low, o));
        }
        const int nb = (lim + L::KEYS - 1) / L::KEYS;
        const int b0 = (int)((long long)nb * x.split / sp.splits), b1 = (int)((long long)nb * (x.split + 1) / sp.splits);
        auto load = [&](int what, int blk) {
            ++asked[what];
            if (!ptx::elect_one()) return;
            ptx::mbar_expect_tx(&bar[what], (uint32_t)L::HALF);
            for (int db = 0; db < DP / 64; ++db)
                kv_load_box(block + what * L::HALF + db * (L::KEYS * 128), what ? &maps.v[side] : &maps.k[side], &bar[what],
                            db * 64, maps.at[side], kvh, blk * L::KEYS, x.cache);
        };
        const int first = b0 + x.wk;
        if (first < b1 && good) {
            load(0, first);
            load(1, first);
        }
        // Query fragments: row g, elements 16 i + 2 j, + 1 and + 8, + 9.
        uint32_t qf[ND][2];
        {
            const int r = x.t.r0 + g;
            const bool in = r < x.t.R;
            const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.c.q) + 2 * j;
            if (in) q += row_token(x.t, a.c.gq, r) * a.c.q_stride + (long long)(x.t.head0 + r % a.c.gq) * a.c.D;
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    qf[i][e] = in && 16 * i + 8 * e < a.c.D ? __ldg((const uint32_t*)(q + 16 * i + 8 * e)) : 0u;
        }
        float o[ND][4];
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        for (int blk = first; blk < b1 && good; blk += x.nwk) {
            const int key0 = blk * L::KEYS;
            good = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(&bar[0], done[0] & 1, RT_WAIT_NS));
            if (!good) break;
            ++done[0];
            float sc[MT][4];
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[t][e] = 0.f;
            const int kr = (lane & 7) + (lane & 8);   // key of this lane's matrix row; its chunk is 2 i + lane / 16
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const int ch = 2 * i + (lane >> 4);
                    uint32_t f[4];
                    ldsm4(f, ks + (ch >> 3) * (L::KEYS * 128) + (16 * t + kr) * 128 + (((ch & 7) ^ (kr & 7)) << 4));
                    kr_mma(sc[t], f[0], f[1], f[2], f[3], qf[i][0], qf[i][1]);
                }
            __syncwarp();
            if (blk + x.nwk < b1) load(0, blk + x.nwk);
            // Keys g, g + 8 of each tile, rows 2 j, 2 j + 1; hidden scores are replaced, whatever they hold.
            float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int key = key0 + 16 * t + g + 8 * e;
                    if (key >= n0) sc[t][2 * e] = -INFINITY;
                    if (key >= n1) sc[t][2 * e + 1] = -INFINITY;
                    x0 = fmaxf(x0, sc[t][2 * e]);
                    x1 = fmaxf(x1, sc[t][2 * e + 1]);
                }
            }
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) {
                x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, d));
                x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, d));
            }
            if (__any_sync(0xffffffffu, x0 > m0 || x1 > m1)) {
                const float y0 = fmaxf(m0, x0), y1 = fmaxf(m1, x1);
                const float a0 = m0 == -INFINITY ? 0.f : kr_ex2((m0 - y0) * a.c2);
                const float a1 = m1 == -INFINITY ? 0.f : kr_ex2((m1 - y1) * a.c2);
                m0 = y0;
                m1 = y1;
                l0 *= a0;
                l1 *= a1;
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    o[i][0] *= a0;
                    o[i][1] *= a1;
                    o[i][2] *= a0;
                    o[i][3] *= a1;
                }
            }
            const float f0 = m0 == -INFINITY ? 0.f : m0, f1 = m1 == -INFINITY ? 0.f : m1;
            uint32_t ph[MT][2], pe[MT][2];
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float p0 = kr_ex2((sc[t][2 * e] - f0) * a.c2), p1 = kr_ex2((sc[t][2 * e + 1] - f1) * a.c2);
                    l0 += p0;
                    l1 += p1;
                    const uint32_t h = kr_pack(p0, p1);
                    const uint32_t r = kr_pack(p0 - __uint_as_float(h << 16), p1 - __uint_as_float(h & 0xffff0000u));
                    ph[t][e] = kr_transpose(h);
                    pe[t][e] = kr_transpose(r);
                }
            good = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(&bar[1], done[1] & 1, RT_WAIT_NS));
            if (!good) break;
            ++done[1];
            const int vr = (lane & 7) + ((lane >> 4) << 3);   // key of this lane's matrix row; its chunk is 2 i + bit 3
            auto values = [&](int t, int i, uint32_t(&f)[4]) {
                const int ch = 2 * i + ((lane >> 3) & 1);
                ldsm4_t(f, vs + (ch >> 3) * (L::KEYS * 128) + (16 * t + vr) * 128 + (((ch & 7) ^ (vr & 7)) << 4));
            };
            // Values of keys from `n` on become zeros, whatever they hold (0 times a NaN is not 0).
            auto mask = [&](int t, int n, uint32_t& lo, uint32_t& hi) {
                const int key = key0 + 16 * t + 2 * j;
                lo = (key < n ? 0xffffu : 0u) | (key + 1 < n ? 0xffff0000u : 0u);
                hi = (key + 8 < n ? 0xffffu : 0u) | (key + 9 < n ? 0xffff0000u : 0u);
            };
            // A block that some rows see only a part of, with an infinity or NaN among its values: row by row over the
            // row's own keys (one row's would reach another).
            bool odd = false;
            if (low < min(key0 + L::KEYS, lim)) {
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    uint32_t lo, hi;
                    mask(t, lim, lo, hi);
                    for (int i = 0; i < ND; ++i) {
                        uint32_t f[4];
                        values(t, i, f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t v = f[e] & (e < 2 ? lo : hi);
                            odd = odd || (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
                        }
                    }
                }
                odd = __any_sync(0xffffffffu, odd);
            }
            auto product = [&](int n, bool cut, int row) {
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    uint32_t lo = ~0u, hi = ~0u;
                    if (cut) mask(t, n, lo, hi);
                    const bool mine = row < 0 || g == row;
                    const uint32_t h0 = mine ? ph[t][0] : 0u, h1 = mine ? ph[t][1] : 0u;
                    const uint32_t e0 = mine ? pe[t][0] : 0u, e1 = mine ? pe[t][1] : 0u;
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        uint32_t f[4];
                        values(t, i, f);
                        kr_mma(o[i], f[0] & lo, f[1] & lo, f[2] & hi, f[3] & hi, h0, h1);
                        kr_mma(o[i], f[0] & lo, f[1] & lo, f[2] & hi, f[3] & hi, e0, e1);
                    }
                }
            };
            if (!odd) {
                product(lim, key0 + L::KEYS > lim, -1);
            } else {
#pragma unroll 1
                for (int r = 0; r < KR_ROWS; ++r) product(__shfl_sync(0xffffffffu, (r & 1) ? n1 : n0, r >> 1), true, r);
            }
            __syncwarp();
            if (blk + x.nwk < b1) load(1, blk + x.nwk);
        }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        // Copies that are still on their way (a wait gave up) land before their memory is used for anything else.
        for (int what = 0; what < 2; ++what)
            for (; done[what] < asked[what]; ++done[what]) (void)ptx::mbar_wait_bounded(&bar[what], done[what] & 1, RT_WAIT_NS);
        __syncthreads();   // every warp is through with its blocks: their memory holds the merge now
        float* f = (float*)rt_smem + warp * MergeSmem<DP>::WARP_FLOATS;
        constexpr int LD = MergeSmem<DP>::LD;
        if (good) {
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) f[(2 * j + (e & 1)) * LD + 16 * i + g + 8 * (e >> 1)] = o[i][e];
        }
        if (g == 0) {
            float* ml = f + KR_ROWS * LD + 4 * j;
            ml[0] = m0;
            ml[1] = l0;
            ml[2] = m1;
            ml[3] = l1;
        }
        merge_and_write<DP, __nv_bfloat16>(a, x, sp, (const float*)rt_smem, warp, lane);
        ptx::fence_proxy_async_smem();   // before the next piece's copies land where the merge was
        __syncthreads();
    }
    if (!good && lane == 0) atomicCAS(a.err, 0, (int)DEV_TIMEOUT_WEIGHTS);
}

// fp32 on CUDA cores: one warp = 8 query rows over 32-key blocks. Scores with a key per lane, the
// values with a lane per four elements of d.
template <int DP>
__global__ void __launch_bounds__(AT_THREADS) k_kv_attend_f32(const __grid_constant__ AttendArgs a) {
    extern __shared__ __align__(16) float kv_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    ptx::grid_dep_launch();
    const Piece x = piece_of(a, blockIdx.x, warp);
    const SidePlan& sp = x.prefix ? a.p : a.o;
    const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
    const int D = a.c.D;
    float* qs = kv_smem + warp / sp.wk * (KR_ROWS * DP);
    if (x.wk == 0) {
        for (int e = lane; e < KR_ROWS * (DP / 4); e += 32) {
            const int rr = e / (DP / 4), d = 4 * (e % (DP / 4)), r = x.t.r0 + rr;
            const float* q = static_cast<const float*>(a.c.q);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < x.t.R && d < D)
                v = *(const float4*)(q + row_token(x.t, a.c.gq, r) * a.c.q_stride + (long long)(x.t.head0 + r % a.c.gq) * D + d);
            *(float4*)(qs + rr * DP + d) = v;
        }
    }
    int n[KR_ROWS], lim = 0;
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r) {
        n[r] = row_seen(a.c, x.prefix, x.cache, x.t, x.t.r0 + r);
        lim = max(lim, n[r]);
    }
    __syncthreads();
    const long long nb = (lim + 31) / 32;
    const int b0 = (int)(nb * x.split / sp.splits), b1 = (int)(nb * (x.split + 1) / sp.splits);
    const float* kbase = (const float*)s.k + x.cache * s.cs + (x.t.head0 / a.c.gq) * s.hs;
    const float* vbase = (const float*)s.v + x.cache * s.cs + (x.t.head0 / a.c.gq) * s.hs;
    constexpr int NI = (DP + 127) / 128;
    float4 o[KR_ROWS][NI];
    float m[KR_ROWS], l[KR_ROWS];
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) o[r][i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int blk = b0 + x.wk; blk < b1; blk += x.nwk) {
        const int key0 = blk * 32, key = key0 + lane;
        float p[KR_ROWS];
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) p[r] = 0.f;
        const float* kp = kbase + (long long)key * s.rs;
        if (key < lim) {
            for (int d = 0; d < D; d += 4) {
                const float4 k = __ldg((const float4*)(kp + d));
#pragma unroll
                for (int r = 0; r < KR_ROWS; ++r) {
                    const float4 q = *(const float4*)(qs + r * DP + d);
                    p[r] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, p[r]))));
                }
            }
        }
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) {
            const float sc = key < n[r] ? p[r] : -INFINITY;
            float mx = sc;
#pragma unroll
            for (int e = 16; e > 0; e >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, e));
            if (mx > m[r]) {
                const float al = m[r] == -INFINITY ? 0.f : exp2f((m[r] - mx) * a.c2);
                m[r] = mx;
                l[r] *= al;
#pragma unroll
                for (int i = 0; i < NI; ++i) o[r][i] = make_float4(o[r][i].x * al, o[r][i].y * al, o[r][i].z * al, o[r][i].w * al);
            }
            p[r] = m[r] == -INFINITY ? 0.f : exp2f((sc - m[r]) * a.c2);
            l[r] += p[r];
        }
        for (int t = 0; t < 32 && key0 + t < lim; ++t) {
            const float* vp = vbase + (long long)(key0 + t) * s.rs;
            float4 v[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int d = 4 * lane + 128 * i;
                v[i] = d < D ? __ldg((const float4*)(vp + d)) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int r = 0; r < KR_ROWS; ++r) {
                const float w = __shfl_sync(0xffffffffu, p[r], t);
                if (key0 + t < n[r]) {   // a hidden value is not even multiplied by zero
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        o[r][i].x = fmaf(w, v[i].x, o[r][i].x);
                        o[r][i].y = fmaf(w, v[i].y, o[r][i].y);
                        o[r][i].z = fmaf(w, v[i].z, o[r][i].z);
                        o[r][i].w = fmaf(w, v[i].w, o[r][i].w);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r)
#pragma unroll
        for (int e = 16; e > 0; e >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], e);
    __syncthreads();   // the queries have been read
    float* f = kv_smem + warp * MergeSmem<DP>::WARP_FLOATS;
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int d = 4 * lane + 128 * i;
            if (d < DP) *(float4*)(f + r * MergeSmem<DP>::LD + d) = o[r][i];
        }
        if (lane == 0) {
            f[KR_ROWS * MergeSmem<DP>::LD + 2 * r] = m[r];
            f[KR_ROWS * MergeSmem<DP>::LD + 2 * r + 1] = l[r];
        }
    }
    merge_and_write<DP, float>(a, x, sp, kv_smem, warp, lane);
}

// Joins the parts of all rows: `wpr` warps (1, 2 or 4) a row, each with every wpr-th part.
template <int DP, typename E>
__global__ void __launch_bounds__(AT_THREADS) k_kv_combine(const __grid_constant__ AttendArgs a, int wpr) {
    __shared__ float4 so[AT_WARPS][RowAcc<DP>::NI][32];
    __shared__ float sl[AT_WARPS];
    constexpr int NI = RowAcc<DP>::NI;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = warp % wpr;
    const long long row = ((long long)blockIdx.x * AT_WARPS + warp) / wpr;
    ptx::grid_dep_wait();
    RowAcc<DP> acc;
    acc.m = -INFINITY;
    acc.l = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) acc.o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < a.rows) join_parts<DP>(a, acc, row, a.p.splits + a.o.splits, first, wpr, lane);
    if (wpr > 1) {
#pragma unroll
        for (int i = 0; i < NI; ++i) so[warp][i][lane] = acc.o[i];
        if (lane == 0) sl[warp] = acc.l;
        __syncthreads();
        if (first != 0) return;
        for (int k = 1; k < wpr; ++k) {
            float4 v[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) v[i] = so[warp + k][i][lane];
            acc.add(1.f, v);
            acc.l += sl[warp + k];
        }
    }
    if (row < a.rows) write_row<DP, E>(a, acc, row, lane);
}

// Rows of partial outputs the workspace holds.
long long ws_rows(const jpi_kv_handle* h) {
    const long long rows = (long long)h->cfg.max_batch * h->cfg.max_tokens * h->H;
    return 2 * rows + 512ll * h->num_sms;
}

// A side's pieces for blocks of `warps` warps: key splits until there are `want` pieces in all, as long as a warp keeps
// `least` keys and the parts fit their half of the workspace.
SidePlan plan_side(const jpi_kv_handle* h, const KvCall& c, bool prefix, int warps, int least, long long want) {
    SidePlan s;
    const KvSide& side = prefix ? c.prefix : c.own;
    if (side.rows == 0) return s;
    const int caches = prefix ? c.groups : c.batch;
    const long long R = (long long)(prefix ? c.batch / c.groups : 1) * c.tokens * c.gq;
    const long long rt = (R + KR_ROWS - 1) / KR_ROWS;
    while (s.wr < warps && s.wr < rt) s.wr *= 2;
    s.wk = warps / s.wr;
    s.tiles = (int)((rt + s.wr - 1) / s.wr);
    const long long blocks = (long long)caches * c.K * s.tiles, rows = (long long)c.batch * c.tokens * c.H;
    const long long room = std::max(1ll, (ws_rows(h) / 2) / rows);
    const long long splits = std::min({want / blocks, room, (long long)(side.rows + least * s.wk - 1) / (least * s.wk)});
    s.splits = (int)std::max(1ll, splits);
    s.blocks = blocks * s.splits;
    return s;
}

template <int DP>
jpi_status launch_dim(jpi_kv_handle* h, const KvCall& c, void* out, float* lse, cudaStream_t st) {
    AttendArgs a = {};
    a.c = c;
    a.c2 = KR_LOG2E * c.scale;
    a.rows = (long long)c.batch * c.tokens * c.H;
    a.po = static_cast<float*>(h->ws);
    a.pml = reinterpret_cast<float2*>(a.po + (size_t)ws_rows(h) * c.D);
    a.lse = lse;
    a.err = h->dev_err;
    int splits = 0;
    const bool tiles = kv_prefix_splits(h, c, std::max(1ll, ws_rows(h) / 2 / a.rows), &splits);
    // The row kernel: on bulk copies where both sides' strides allow them.
    KvMapDims md[2];
    const bool copies = h->bf16 && c.D >= 64 && kv_maps_available() &&
                        (tiles || c.prefix.rows == 0 || kv_map_dims(c.prefix, c.K, c.D, c.groups, &md[0])) &&
                        (c.own.rows == 0 || kv_map_dims(c.own, c.K, c.D, c.batch, &md[1]));
    const int warps = copies ? RT_WARPS : AT_WARPS, least = copies ? RtSmem<DP>::KEYS : h->bf16 ? KR_KEYS : 32;
    const long long want = 2ll * h->num_sms;
    a.p = plan_side(h, c, true, warps, least, want);
    a.o = plan_side(h, c, false, warps, least, want);
    if (tiles) {
        a.p.blocks = 0;
        a.p.splits = splits;
    }
    const int parts = a.p.splits + a.o.splits;
    const long long pieces = a.p.blocks + a.o.blocks;
    if (pieces > 0x7fffffffll) {
        set_error("the call needs more than 2^31 blocks");
        return JPI_ERR_SHAPE;
    }
    if (pieces > 0) {
        AttendArgs r = a;
        if (parts == 1) r.out = out;
        if (copies) {
            RtMaps m = {};
            for (int i = 0; i < 2; ++i) {
                const KvSide& s = i ? c.own : c.prefix;
                if (s.rows == 0 || (i == 0 && tiles)) continue;
                if (!kv_make_map(md[i], s.k, c.D, RtSmem<DP>::KEYS, &m.k[i]) || !kv_make_map(md[i], s.v, c.D, RtSmem<DP>::KEYS, &m.v[i])) {
                    set_error("cuTensorMapEncodeTiled refused the %s", i ? "own rows" : "prefix");
                    return JPI_ERR_CUDA;
                }
                m.at[i] = make_int3(md[i].at_head, md[i].at_row, md[i].at_cache);
            }
            const long long most = (tiles ? 2ll : 6ll) * h->num_sms;
            JPI_TRY(kv_start(k_kv_attend_rows<DP>, std::min(pieces, most), RT_THREADS, RtSmem<DP>::BYTES, false, st, m, r));
        } else if (h->bf16) {
            JPI_TRY(kv_start(k_kv_attend_mma<DP>, pieces, AT_THREADS, MergeSmem<DP>::BYTES, false, st, r));
        } else {
            JPI_TRY(kv_start(k_kv_attend_f32<DP>, pieces, AT_THREADS, MergeSmem<DP>::BYTES, false, st, r));
        }
    }
    if (tiles) JPI_TRY(launch_kv_prefix_t5(h, c, splits, a.po, a.pml, pieces > 0, st));
    if (parts == 1 && pieces > 0) return JPI_OK;
    a.out = out;
    const int wpr = parts > 16 ? 4 : parts > 4 ? 2 : 1;
    const long long grid = (a.rows * wpr + AT_WARPS - 1) / AT_WARPS;
    return h->bf16 ? kv_start(k_kv_combine<DP, __nv_bfloat16>, grid, AT_THREADS, 0, true, st, a, wpr)
                   : kv_start(k_kv_combine<DP, float>, grid, AT_THREADS, 0, true, st, a, wpr);
}

template <int DP>
jpi_status prepare_dim() {
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_mma<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, MergeSmem<DP>::BYTES));
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_f32<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, MergeSmem<DP>::BYTES));
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_rows<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, RtSmem<DP>::BYTES));
    // All of its loads go to shared memory, and the 128-row tiles need the SM set up for the most of it.
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_rows<DP>, cudaFuncAttributePreferredSharedMemoryCarveout,
                                      cudaSharedmemCarveoutMaxShared));
    return JPI_OK;
}

}  // namespace

size_t kv_attend_ws_bytes(const jpi_kv_handle* h) {
    return (size_t)ws_rows(h) * (h->D * sizeof(float) + sizeof(float2));
}

jpi_status kv_attend_prepare(jpi_kv_handle* h) {
    JPI_TRY(kv_prefix_prepare(h));
    return h->D <= 64 ? prepare_dim<64>() : h->D <= 128 ? prepare_dim<128>() : prepare_dim<256>();
}

jpi_status launch_kv_attend(jpi_kv_handle* h, const KvCall& c, void* out, float* lse, cudaStream_t st) {
    return h->D <= 64 ? launch_dim<64>(h, c, out, lse, st)
                      : h->D <= 128 ? launch_dim<128>(h, c, out, lse, st) : launch_dim<256>(h, c, out, lse, st);
}

}  // namespace jpi
