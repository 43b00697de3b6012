// Attention over windows of a cache, in the handle's type or in 8 bits (jpi_kv_attend_window, jpi_kv8_attend).
//
//   o_r = sum_j p_rj v_j,  p_rj = exp(s_rj - lse_r),  s_rj = scale q_r . k_j,
// j over the rows that the token of query row r sees (kv_span.h); in 8 bits k_j and v_j are codes times the power of two of
// their block and head.
//
// Query rows of one request and KV head form tiles of 8 (kv_rows.cuh), a tile's rows of the cache are those that one of
// its tokens sees, and every part (a range of them) leaves partial rows that are joined as in kv_attend.cu.

#include "kv_attend.h"
#include "kv_parts.cuh"
#include "kv8.cuh"
#include "kv_span.cuh"

#include <algorithm>

namespace jpi {
namespace {

struct SpanArgs {
    AttendArgs a;
    KvSpan s;
};

// Four elements of a cache's row as fp32.
struct Code8 { uint8_t code; };
template <typename T>
__device__ __forceinline__ float4 four(const T* p);
template <>
__device__ __forceinline__ float4 four<float>(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
template <>
__device__ __forceinline__ float4 four<__nv_bfloat16>(const __nv_bfloat16* p) {
    const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u));
}
template <>
__device__ __forceinline__ float4 four<Code8>(const Code8* p) {
    float z[4];
    kv8_values(__ldg(reinterpret_cast<const uint32_t*>(p)), z);
    return make_float4(z[0], z[1], z[2], z[3]);
}

// On CUDA cores: a warp takes 8 query rows over blocks of 32 keys, scores with a key per lane, values with a lane per four
// elements of d; the warps of a block take different row tiles or different keys of one.
template <int DP, typename E, typename T>
__global__ void __launch_bounds__(AT_THREADS, DP == 256 ? 2 : 3) k_kv_span_cc(const __grid_constant__ SpanArgs g) {
    extern __shared__ __align__(16) float kv_smem[];
    const AttendArgs& a = g.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Piece x = piece_of(a, blockIdx.x, warp);
    const SidePlan& sp = a.o;
    const KvSide& s = a.c.own;
    const int D = a.c.D;
    float* qs = kv_smem + warp / sp.wk * (KR_ROWS * DP);
    const int wk = warp % sp.wk;
    if (wk == 0) {
        for (int e = lane; e < KR_ROWS * (DP / 4); e += 32) {
            const int r = x.t.r0 + e / (DP / 4), d = 4 * (e % (DP / 4));
            *(float4*)(qs + 4 * e) = r < x.t.R && d < D ? four<E>(static_cast<const E*>(a.c.q) + row_query(a.c, x.t, r) + d)
                                                        : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    int n[KR_ROWS], lim = 0, first = 0x7fffffff;
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r) {
        n[r] = row_seen(a.c, false, x.cache, x.t, x.t.r0 + r);
        lim = max(lim, n[r]);
        if (n[r] > 0) first = min(first, span_first(g.s, n[r]));
    }
    __syncthreads();
    const SpanBlocks<32> blocks(g.s, lim, first);
    const int b0 = (int)((long long)blocks.count * x.split / sp.splits), b1 = (int)((long long)blocks.count * (x.split + 1) / sp.splits);
    const T* kbase = (const T*)s.k + x.cache * s.cs + x.kvh * s.hs;
    const T* vbase = (const T*)s.v + x.cache * s.cs + x.kvh * s.hs;
    const long long scales = ((long long)x.cache * a.c.K + x.kvh) * g.s.nblk;
    constexpr bool HELD8 = sizeof(T) == 1;
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
    for (int blk = b0 + wk; blk < b1; blk += sp.wk) {
        const int key0 = blocks.row(blk), key = key0 + lane;
        float p[KR_ROWS];
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) p[r] = 0.f;
        const bool live = span_sees(g.s, key, lim, first);   // by some row of the tile
        const T* kp = kbase + (long long)key * s.rs;
        for (int d = 0; d < D; d += 4) {
            const float4 k = live ? four<T>(kp + d) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int r = 0; r < KR_ROWS; ++r) {
                const float4 q = *(const float4*)(qs + r * DP + d);
                p[r] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, p[r]))));
            }
        }
        float ks = 1.f, vs = 1.f;
        if (HELD8 && live) {
            ks = kv8_scale(g.s.ks[scales + (key >> g.s.n_log2)]);
            vs = kv8_scale(g.s.vs[scales + (key >> g.s.n_log2)]);
        }
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) {
            const float sc = span_sees(g.s, key, n[r], span_first(g.s, n[r])) ? p[r] * ks : -INFINITY;
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
            p[r] = exp2f((sc - (m[r] == -INFINITY ? 0.f : m[r])) * a.c2);   // (of -inf 0, of NaN NaN)
            l[r] += p[r];
        }
        for (int t = 0; t < 32 && key0 + t < lim; ++t) {
            if (!span_sees(g.s, key0 + t, lim, first)) continue;   // (the same for the warp)
            const float by = HELD8 ? __shfl_sync(0xffffffffu, vs, t) : 1.f;
            float4 v[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int d = 4 * lane + 128 * i;
                v[i] = d < D ? four<T>(vbase + (long long)(key0 + t) * s.rs + d) : make_float4(0.f, 0.f, 0.f, 0.f);
                if (HELD8) v[i] = make_float4(v[i].x * by, v[i].y * by, v[i].z * by, v[i].w * by);
            }
#pragma unroll
            for (int r = 0; r < KR_ROWS; ++r) {
                const float w = __shfl_sync(0xffffffffu, p[r], t);
                if (!span_sees(g.s, key0 + t, n[r], span_first(g.s, n[r]))) continue;   // a hidden value is not even multiplied by zero
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
    __syncthreads();   // the queries have been read
    float* f = kv_smem + warp * MergeSmem<DP>::WARP_FLOATS;
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r) {
#pragma unroll
        for (int e = 16; e > 0; e >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], e);
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
    merge_and_write<DP, E>(a, x, sp, kv_smem, warp, lane);
}

// Pieces for blocks of `warps` warps that take blocks of `step` keys: splits of the rows that a tile can see, while each
// warp keeps one and the parts fit the workspace, to `want` blocks in all.
SidePlan plan_span(const jpi_kv_handle* h, const KvCall& c, const KvSpan& sn, int warps, int step, long long want) {
    SidePlan s;
    const long long R = (long long)c.tokens * c.gq, rt = (R + KR_ROWS - 1) / KR_ROWS;
    while (s.wr < warps && s.wr < rt) s.wr *= 2;
    s.wk = warps / s.wr;
    s.tiles = (int)((rt + s.wr - 1) / s.wr);
    // Rows of the cache that a tile's tokens see, and the ends of their blocks.
    const long long toks = std::min<long long>(c.tokens, (KR_ROWS + c.gq - 1) / c.gq + 1);
    const long long rows = std::min<long long>(c.own.rows, (long long)sn.window + toks + std::min(sn.sink, c.own.rows) + 2 * step);
    const long long blocks = (long long)c.batch * c.K * s.tiles, all = (long long)c.batch * c.tokens * c.H;
    const long long room = std::max(1ll, ws_rows(h) / all);
    s.splits = (int)std::max(1ll, std::min({want / blocks, (rows + step * s.wk - 1) / (step * s.wk), room}));
    s.blocks = blocks * s.splits;
    s.by_splits = KvDiv((uint32_t)s.splits);
    s.by_tiles = KvDiv((uint32_t)s.tiles);
    return s;
}

template <int DP, typename E>
jpi_status launch_dim(jpi_kv_handle* h, const KvCall& c, const KvSpan& sn, void* out, float* lse, cudaStream_t st) {
    SpanArgs g = {};
    AttendArgs& a = g.a;
    g.s = sn;
    a.c = c;
    a.c2 = KR_LOG2E * c.scale;
    a.rows = (long long)c.batch * c.tokens * c.H;
    a.po = static_cast<float*>(h->ws);
    a.pml = reinterpret_cast<float2*>(a.po + (size_t)ws_rows(h) * c.D);
    a.lse = lse;
    a.o = plan_span(h, c, sn, AT_WARPS, 32, 2ll * h->num_sms);
    a.p.splits = 0;
    a.parts = a.o.splits;
    if (a.o.blocks > 0x7fffffffll) {
        set_error("the call needs more than 2^31 blocks");
        return JPI_ERR_SHAPE;
    }
    if (a.parts == 1) a.out = out;
    JPI_TRY(kv_start(sn.ks ? k_kv_span_cc<DP, E, Code8> : k_kv_span_cc<DP, E, E>, dim3((unsigned)a.o.blocks), AT_THREADS,
                     MergeSmem<DP>::BYTES, false, st, g));
    return a.parts == 1 ? JPI_OK : launch_kv_combine(h, c, a.parts, out, lse, st);
}

template <int DP, typename E>
jpi_status prepare_dim() {
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_span_cc<DP, E, E>, cudaFuncAttributeMaxDynamicSharedMemorySize, MergeSmem<DP>::BYTES));
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_span_cc<DP, E, Code8>, cudaFuncAttributeMaxDynamicSharedMemorySize, MergeSmem<DP>::BYTES));
    return JPI_OK;
}

template <typename E>
jpi_status launch_type(jpi_kv_handle* h, const KvCall& c, const KvSpan& s, void* out, float* lse, cudaStream_t st) {
    return h->D <= 64 ? launch_dim<64, E>(h, c, s, out, lse, st)
                      : h->D <= 128 ? launch_dim<128, E>(h, c, s, out, lse, st) : launch_dim<256, E>(h, c, s, out, lse, st);
}
template <typename E>
jpi_status prepare_type(const jpi_kv_handle* h) {
    return h->D <= 64 ? prepare_dim<64, E>() : h->D <= 128 ? prepare_dim<128, E>() : prepare_dim<256, E>();
}

}  // namespace

jpi_status kv_span_prepare(jpi_kv_handle* h) { return h->bf16 ? prepare_type<__nv_bfloat16>(h) : prepare_type<float>(h); }

jpi_status launch_kv_span(jpi_kv_handle* h, const KvCall& c, const KvSpan& s, void* out, float* lse, cudaStream_t st) {
    return h->bf16 ? launch_type<__nv_bfloat16>(h, c, s, out, lse, st) : launch_type<float>(h, c, s, out, lse, st);
}

}  // namespace jpi
