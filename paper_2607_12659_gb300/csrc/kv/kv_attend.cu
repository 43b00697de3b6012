// Attention of a batch over shared prefixes and own rows (jpi_kv_attend).
//
//   o_r = sum_j p_rj v_j,  p_rj = exp(s_rj - lse_r),  s_rj = scale q_r . k_j,
// j over the first prefix_len rows of the run's prefix and then the first `seen` rows of the request's own
// cache. A prefix is read once for all its requests: their query rows are one matrix.
//
// The softmax is computed in parts: every part (a range of keys of one side) keeps a running maximum m and
// sum l per row and an unnormalised output, all fp32, and k_kv_combine joins them,
//   o = sum_s w_s O_s / sum_s w_s l_s,  w_s = exp(scale (m_s - M)),
// in part order, so that a result does not depend on which block finished first. A part that saw no key
// has m = -inf and weighs nothing; a row of only such parts is zero. Maxima are those of the unscaled
// products, and the difference is scaled, not the product: log2(e) times a score near the type's largest
// values would overflow.

#include "kv_rows.cuh"
#include "kv_attend.h"

#include <algorithm>

namespace jpi {
namespace {

constexpr int AT_WARPS = 8;
constexpr int AT_THREADS = 32 * AT_WARPS;

// How one side is dealt to blocks: `wr` warps of a block take different row tiles and 8 / wr different keys.
struct SidePlan {
    int wr = 1, wk = AT_WARPS;
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
};

// The block's piece of work: side, cache, KV head, row tile and key split.
struct Piece {
    bool prefix;
    int cache, split, part;
    RowTile t;
    int wk, nwk;
};
__device__ __forceinline__ Piece piece_of(const AttendArgs& a, int warp) {
    Piece x;
    long long i = blockIdx.x;
    x.prefix = i < a.p.blocks;
    if (!x.prefix) i -= a.p.blocks;
    const SidePlan& s = x.prefix ? a.p : a.o;
    x.split = (int)(i % s.splits);
    i /= s.splits;
    const int tile = (int)(i % s.tiles);
    i /= s.tiles;
    const int kvh = (int)(i % a.c.K);
    x.cache = (int)(i / a.c.K);
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

// Shared memory of one warp's share of the merge: 8 rows of DP outputs, then (m, l) per row.
template <int DP>
struct MergeSmem {
    static constexpr int LD = DP + 4;   // the row pad spreads the rows over the banks
    static constexpr int WARP_FLOATS = KR_ROWS * LD + 2 * KR_ROWS;
    static constexpr int BYTES = AT_WARPS * WARP_FLOATS * 4;
};

// Joins the key warps of each row tile (their outputs and (m, l) are in shared memory) and writes the part.
template <int DP>
__device__ __forceinline__ void merge_and_write(const AttendArgs& a, const Piece& x, const SidePlan& s, float* sm, int warp,
                                                int lane) {
    using M = MergeSmem<DP>;
    __syncthreads();
    // Every warp takes rows (its index among the key warps) + n nwk of its row tile.
    const float* tile = sm + (warp / s.wk) * s.wk * M::WARP_FLOATS;
    for (int rr = x.wk; rr < KR_ROWS; rr += x.nwk) {
        const int r = x.t.r0 + rr;
        if (r >= x.t.R) continue;
        float m = -INFINITY;
        for (int k = 0; k < x.nwk; ++k) m = fmaxf(m, tile[k * M::WARP_FLOATS + KR_ROWS * M::LD + 2 * rr]);
        float l = 0.f;
        const long long row = (long long)x.part * a.rows + row_index(x.t, a.c.gq, a.c.H, r);
        float4 o[DP / 128 + (DP % 128 != 0)];
#pragma unroll
        for (int i = 0; i < (DP + 127) / 128; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < x.nwk; ++k) {
            const float* f = tile + k * M::WARP_FLOATS;
            const float mk = f[KR_ROWS * M::LD + 2 * rr];
            const float w = mk == -INFINITY ? 0.f : kr_ex2((mk - m) * a.c2);
            l += w * f[KR_ROWS * M::LD + 2 * rr + 1];
#pragma unroll
            for (int i = 0; i < (DP + 127) / 128; ++i) {
                const int d = 4 * lane + 128 * i;
                if (d < DP) {
                    const float4 v = *(const float4*)(f + rr * M::LD + d);
                    o[i].x = fmaf(w, v.x, o[i].x);
                    o[i].y = fmaf(w, v.y, o[i].y);
                    o[i].z = fmaf(w, v.z, o[i].z);
                    o[i].w = fmaf(w, v.w, o[i].w);
                }
            }
        }
        if (lane == 0) a.pml[row] = make_float2(m, l);
        if (m != -INFINITY) {
#pragma unroll
            for (int i = 0; i < (DP + 127) / 128; ++i) {
                const int d = 4 * lane + 128 * i;
                if (d < a.c.D) *(float4*)(a.po + row * a.c.D + d) = o[i];
            }
        }
    }
}

// bf16, any head dim to DP: one warp = 8 query rows over the 16-key blocks wk, wk + nwk, .. of the split.
// Probabilities enter the second product as two bf16 terms (the rounded value and what the rounding left), so
// that its error stays that of fp32 sums: the products are bound by the loads of keys and values, and the
// second term costs no time there.
template <int DP>
__global__ void __launch_bounds__(AT_THREADS, 1) k_kv_attend_mma(const __grid_constant__ AttendArgs a) {
    extern __shared__ __align__(16) float kv_smem[];
    constexpr int NC = DP / 32;    // chunk groups of a key
    constexpr int NV = DP / 64;    // chunk groups of a value row
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, j = lane & 3;
    const Piece x = piece_of(a, warp);
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
    merge_and_write<DP>(a, x, sp, kv_smem, warp, lane);
}

// fp32 on CUDA cores: one warp = 8 query rows over 32-key blocks. Scores with a key per lane, the
// values with a lane per four elements of d.
template <int DP>
__global__ void __launch_bounds__(AT_THREADS) k_kv_attend_f32(const __grid_constant__ AttendArgs a) {
    extern __shared__ __align__(16) float kv_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Piece x = piece_of(a, warp);
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
    merge_and_write<DP>(a, x, sp, kv_smem, warp, lane);
}

// Joins the parts of a row: one block per row, D / 4 threads per group of parts.
constexpr int CB_THREADS = 128;
template <typename E>
__global__ void __launch_bounds__(CB_THREADS) k_kv_combine(const float* __restrict__ po, const float2* __restrict__ pml,
                                                           long long rows, int parts, int D, float scale, E* out, float* lse) {
    extern __shared__ __align__(16) float kv_smem[];   // [parts] weights, then [groups][D]
    __shared__ float red[CB_THREADS / 32];
    const int t = threadIdx.x;
    const long long row = blockIdx.x;
    float m = -INFINITY;
    for (int p = t; p < parts; p += CB_THREADS) m = fmaxf(m, pml[p * rows + row].x);
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, e));
    if ((t & 31) == 0) red[t >> 5] = m;
    __syncthreads();
    m = red[0];
#pragma unroll
    for (int i = 1; i < CB_THREADS / 32; ++i) m = fmaxf(m, red[i]);
    __syncthreads();
    float l = 0.f;
    for (int p = t; p < parts; p += CB_THREADS) {
        const float2 v = pml[p * rows + row];
        const float w = v.x == -INFINITY ? 0.f : kr_ex2((v.x - m) * (KR_LOG2E * scale));
        kv_smem[p] = w;
        l += w * v.y;
    }
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) l += __shfl_xor_sync(0xffffffffu, l, e);
    if ((t & 31) == 0) red[t >> 5] = l;
    __syncthreads();
    l = red[0];
#pragma unroll
    for (int i = 1; i < CB_THREADS / 32; ++i) l += red[i];
    if (t == 0 && lse) lse[row] = m == -INFINITY ? -INFINITY : fmaf(m, scale, logf(l));
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int lanes = D / 4, groups = CB_THREADS / lanes, gr = t / lanes, d = 4 * (t % lanes);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (gr < groups)
        for (int p = gr; p < parts; p += groups) {
            const float w = kv_smem[p];
            if (w > 0.f) {
                const float4 v = *(const float4*)(po + (p * rows + row) * D + d);
                o.x = fmaf(w, v.x, o.x);
                o.y = fmaf(w, v.y, o.y);
                o.z = fmaf(w, v.z, o.z);
                o.w = fmaf(w, v.w, o.w);
            }
        }
    float4* sums = reinterpret_cast<float4*>(kv_smem + ((parts + 3) & ~3));
    if (groups > 1) {
        if (gr < groups) sums[gr * lanes + t % lanes] = o;
        __syncthreads();
        if (gr == 0)
            for (int i = 1; i < groups; ++i) {
                const float4 v = sums[i * lanes + t];
                o = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
            }
    }
    if (gr == 0) {
        if constexpr (sizeof(E) == 2)
            *(uint2*)(out + row * D + d) = make_uint2(kr_pack(o.x * inv, o.y * inv), kr_pack(o.z * inv, o.w * inv));
        else
            *(float4*)(out + row * D + d) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    }
}

// Rows of partial outputs the workspace holds.
long long ws_rows(const jpi_kv_handle* h) {
    const long long rows = (long long)h->cfg.max_batch * h->cfg.max_tokens * h->H;
    return 2 * rows + 512ll * h->num_sms;
}

// A side's key splits: enough blocks for the SMs, as long as a block keeps at least `least` keys and the parts
// fit their half of the workspace.
SidePlan plan_side(const jpi_kv_handle* h, const KvCall& c, bool prefix, int least) {
    SidePlan s;
    const KvSide& side = prefix ? c.prefix : c.own;
    if (side.rows == 0) return s;
    const int caches = prefix ? c.groups : c.batch;
    const long long R = (long long)(prefix ? c.batch / c.groups : 1) * c.tokens * c.gq;
    const long long rt = (R + KR_ROWS - 1) / KR_ROWS;
    s.wr = 1;
    while (s.wr < AT_WARPS && s.wr < rt) s.wr *= 2;
    s.wk = AT_WARPS / s.wr;
    s.tiles = (int)((rt + s.wr - 1) / s.wr);
    const long long blocks = (long long)caches * c.K * s.tiles, rows = (long long)c.batch * c.tokens * c.H;
    const long long room = std::max(1ll, (ws_rows(h) / 2) / rows);
    long long splits = (h->num_sms + blocks - 1) / blocks;
    splits = std::min({splits, room, (long long)(side.rows + least * s.wk - 1) / (least * s.wk)});
    s.splits = (int)std::max(1ll, splits);
    s.blocks = blocks * s.splits;
    return s;
}

template <int DP>
jpi_status launch_parts(const jpi_kv_handle* h, const AttendArgs& a, cudaStream_t st) {
    const unsigned grid = (unsigned)(a.p.blocks + a.o.blocks);
    if (h->bf16)
        k_kv_attend_mma<DP><<<grid, AT_THREADS, MergeSmem<DP>::BYTES, st>>>(a);
    else
        k_kv_attend_f32<DP><<<grid, AT_THREADS, MergeSmem<DP>::BYTES, st>>>(a);
    JPI_CUDA_TRY(cudaGetLastError());
    return JPI_OK;
}

template <int DP>
jpi_status prepare_dim() {
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_mma<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, MergeSmem<DP>::BYTES));
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_f32<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, MergeSmem<DP>::BYTES));
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
    AttendArgs a;
    a.c = c;
    a.p = plan_side(h, c, true, h->bf16 ? KR_KEYS : 32);
    a.o = plan_side(h, c, false, h->bf16 ? KR_KEYS : 32);
    a.c2 = KR_LOG2E * c.scale;
    a.rows = (long long)c.batch * c.tokens * c.H;
    a.po = static_cast<float*>(h->ws);
    a.pml = reinterpret_cast<float2*>(a.po + (size_t)ws_rows(h) * c.D);
    // Many rows on one prefix go to the tensor-core tiles, its parts first.
    int splits = 0;
    const bool tiles = kv_prefix_splits(h, c, std::max(1ll, ws_rows(h) / 2 / a.rows), &splits);
    if (tiles) {
        a.p.blocks = 0;
        a.p.splits = splits;
    }
    if (a.p.blocks + a.o.blocks > 0x7fffffffll) {
        set_error("the call needs more than 2^31 blocks");
        return JPI_ERR_SHAPE;
    }
    if (tiles) JPI_TRY(launch_kv_prefix_t5(h, c, splits, a.po, a.pml, st));
    if (a.p.blocks + a.o.blocks > 0)
        JPI_TRY(h->D <= 64 ? launch_parts<64>(h, a, st) : h->D <= 128 ? launch_parts<128>(h, a, st) : launch_parts<256>(h, a, st));
    const int parts = a.p.splits + a.o.splits;
    const size_t smem = (size_t)((parts + 3) & ~3) * 4 + CB_THREADS * 16;
    if (h->bf16)
        k_kv_combine<__nv_bfloat16><<<(unsigned)a.rows, CB_THREADS, smem, st>>>(a.po, a.pml, a.rows, parts, c.D, c.scale,
                                                                                (__nv_bfloat16*)out, lse);
    else
        k_kv_combine<float><<<(unsigned)a.rows, CB_THREADS, smem, st>>>(a.po, a.pml, a.rows, parts, c.D, c.scale, (float*)out, lse);
    JPI_CUDA_TRY(cudaGetLastError());
    return JPI_OK;
}

}  // namespace jpi
