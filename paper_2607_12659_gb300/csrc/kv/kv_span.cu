// Attention over windows of a cache, in the handle's type or in 8 bits (jpi_kv_attend_window, jpi_kv8_attend).
//
//   o_r = sum_j p_rj v_j,  p_rj = exp(s_rj - lse_r),  s_rj = scale q_r . k_j,
// j over the rows that the token of query row r sees (kv_span.h); in 8 bits k_j and v_j are codes times the power of two of
// their block and head.
//
// Query rows of one request and KV head form tiles of 8 (kv_rows.cuh), a tile's rows of the cache are the first `sink` and those from its
// windows' lowest row to its largest count (SpanBlocks), and every part (a range of them) leaves partial rows that are joined as in kv_attend.cu.

#include "kv_attend.h"
#include "kv_parts.cuh"
#include "kv8.cuh"
#include "kv_pair.cuh"
#include "kv_span.cuh"

#include <algorithm>
#include <type_traits>

namespace jpi {
namespace {

struct SpanArgs {
    AttendArgs a;
    KvSpan s;
};

// A cache's elements as they are loaded and as fp32: four of the values, a run of a key.
struct Code8 { uint8_t code; };
template <typename T>
struct Held;
template <>
struct Held<float> {
    using Four = float4;
    __device__ static __forceinline__ Four four(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
    __device__ static __forceinline__ Four none() { return make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ static __forceinline__ float4 value(Four x) { return x; }
    // Elements of a key that are on their way together, and how they are used.
    static constexpr int RUN = 16;
    struct Run { float4 x[4]; };
    __device__ static __forceinline__ void load(Run& r, const float* p, int n) {   // n: left of the row
#pragma unroll
        for (int i = 0; i < 4; ++i) r.x[i] = 4 * i < n ? four(p + 4 * i) : none();
    }
    __device__ static __forceinline__ float4 part(const Run& r, int i) { return r.x[i]; }
};
template <>
struct Held<Code8> {
    using Four = uint32_t;
    __device__ static __forceinline__ Four four(const Code8* p) { return __ldg(reinterpret_cast<const uint32_t*>(p)); }
    __device__ static __forceinline__ Four none() { return 0; }
    __device__ static __forceinline__ float4 value(Four x) {
        float z[4];
        kv8_values(x, z);
        return make_float4(z[0], z[1], z[2], z[3]);
    }
    static constexpr int RUN = 16;
    struct Run { uint4 x; };
    __device__ static __forceinline__ void load(Run& r, const Code8* p, int) { r.x = __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ static __forceinline__ float4 part(const Run& r, int i) { return value(i == 0 ? r.x.x : i == 1 ? r.x.y : i == 2 ? r.x.z : r.x.w); }
};

constexpr int SR_RANKS = 8;   // most blocks of a cluster, as in the handle's table
// Most blocks of keys for a warp of a cluster. Microseconds of one launch and of two, bf16 and 8 bits, single tokens over one KV head
// of 256: 300 keys 6.7 and 8.4, 8.0 and 8.9 for one request, 8.4 and 8.9, 8.7 and 10.0 for 16; 867 keys 7.8 and 8.3, 8.5 and 9.3 for one; 2000
// keys (four blocks, two) 9.3 and 9.1, 9.6 and 10.6 for one, 9.6 and 11.1, 9.9 and 12.2 for eight; 4000 keys (eight, four) 12.0 and 9.6, 11.8 and
// 11.0 for one, 12.1 and 11.7, 11.9 and 13.1 for four. (On the host a launch less is 2 us less.)
constexpr int SR_JOIN_BLOCKS = 4;

// Joins the parts of a tile of 8 query rows that the warps of a cluster's blocks hold in shared memory, and writes the result: each
// block its own warps' first, then every block some of the rows over all blocks. A warp's part is laid out as in MergeSmem, PART bytes
// from the one before; behind them lie the block's joined rows and their (m, l).
template <int DP, typename E, int TEAM, int PART>
struct JoinSmem {
    static constexpr int ROWS = TEAM * PART, ML = ROWS + KR_ROWS * DP * 4, BYTES = ML + KR_ROWS * 8;
    static_assert(PART % 16 == 0 && BYTES <= 227 * 1024, "fits an SM");
};
template <int DP, typename E, int TEAM, int PART>
__device__ __forceinline__ void join_cluster(const AttendArgs& a, const Piece& x, int ranks, uint8_t* block, int warp, int lane) {
    using L = JoinSmem<DP, E, TEAM, PART>;
    constexpr int LD = MergeSmem<DP>::LD, NI = (DP + 127) / 128;
    float* const joined = reinterpret_cast<float*>(block + L::ROWS);
    float2* const ml = reinterpret_cast<float2*>(block + L::ML);
    auto part = [&](int k) { return reinterpret_cast<const float*>(block + k * PART); };
    auto weight = [&](float m, float most) { return m == -INFINITY ? 0.f : kr_ex2((m - most) * a.c2); };
    for (int r = warp; r < KR_ROWS; r += TEAM) {
        float2 p[TEAM];
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int k = 0; k < TEAM; ++k) {
            p[k] = *(const float2*)(part(k) + KR_ROWS * LD + 2 * r);
            m = fmaxf(m, p[k].x);
        }
        float4 o[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < TEAM; ++k) {
            if (p[k].y == 0.f) continue;
            const float w = weight(p[k].x, m);
            l = fmaf(w, p[k].y, l);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int d = 4 * lane + 128 * i;
                if (d >= DP) continue;
                const float4 v = *(const float4*)(part(k) + r * LD + d);
                o[i] = make_float4(fmaf(w, v.x, o[i].x), fmaf(w, v.y, o[i].y), fmaf(w, v.z, o[i].z), fmaf(w, v.w, o[i].w));
            }
        }
        if (ranks == 1) {
            if (x.t.r0 + r < x.t.R) {
                RowAcc<DP> row;
#pragma unroll
                for (int i = 0; i < NI; ++i) row.o[i] = o[i];
                row.m = m;
                row.l = l;
                write_row<DP, E>(a, row, row_index(a.c, x.t, x.t.r0 + r), 0, lane);
            }
            continue;
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int d = 4 * lane + 128 * i;
            if (d < DP) *(float4*)(joined + r * DP + d) = o[i];
        }
        if (lane == 0) ml[r] = make_float2(m, l);
    }
    if (ranks == 1) return;
    __syncwarp();
    ptx::cluster_sync_all();
    for (int r = (int)ptx::cluster_rank(); r < KR_ROWS; r += ranks) {
        if (x.t.r0 + r >= x.t.R) continue;
        const long long row = row_index(a.c, x.t, x.t.r0 + r);
        for (int d = 2 * (int)threadIdx.x; d < a.c.D; d += 64 * TEAM) {
            float2 p[SR_RANKS], v[SR_RANKS];
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int k = 0; k < SR_RANKS; ++k) {
                p[k] = make_float2(-INFINITY, 0.f);
                v[k] = make_float2(0.f, 0.f);
                if (k < ranks) {
                    p[k] = ptx::dsmem_ld_f2(ptx::dsmem_map(ptx::smem_u32(ml + r), (uint32_t)k));
                    v[k] = ptx::dsmem_ld_f2(ptx::dsmem_map(ptx::smem_u32(joined + r * DP + d), (uint32_t)k));
                }
            }
#pragma unroll
            for (int k = 0; k < SR_RANKS; ++k) m = fmaxf(m, p[k].x);
            float2 o = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < SR_RANKS; ++k) {
                if (p[k].y == 0.f) continue;
                const float w = weight(p[k].x, m);
                l = fmaf(w, p[k].y, l);
                o = make_float2(fmaf(w, v[k].x, o.x), fmaf(w, v[k].y, o.y));
            }
            const float inv = inverse_sum(l);
            E* const out = static_cast<E*>(a.out) + row * a.c.D + d;
            if constexpr (sizeof(E) == 2) *(uint32_t*)out = kr_pack(o.x * inv, o.y * inv);
            else *(float2*)out = make_float2(o.x * inv, o.y * inv);
            if (d == 0 && a.lse) a.lse[row] = log_sum(m, l, a.c.scale);
        }
    }
    __syncwarp();
    ptx::cluster_sync_all();   // every block's rows have been read
}

// fp32, on CUDA cores: a warp takes 8 query rows over blocks of 32 keys, scores with a key per lane, values with a lane per four
// elements of d; the warps of a block take different row tiles or different keys of one. What bounds it is latency: a block's
// loads, its products and 2^x follow one another. So a key's next elements, and the next values, are on their way while these
// are used (4 requests of 9 tokens with windows of 300 keys took 22 us with loads one by one), and the values' product reads a key's eight
// probabilities from shared memory and tests nothing where all that a row is given is finite (17 us, and 12 in one launch).
template <int DP>
using CcJoin = JoinSmem<DP, float, AT_WARPS, MergeSmem<DP>::WARP_FLOATS * 4>;
template <int DP, bool JOIN>
struct CcSmem {
    static constexpr int P_OFF = JOIN ? CcJoin<DP>::BYTES : MergeSmem<DP>::BYTES;   // [warp][32 keys][8 rows] probabilities
    static constexpr int BYTES = P_OFF + AT_WARPS * 32 * KR_ROWS * 4;
};
template <int DP, typename T, bool JOIN>
__global__ void __launch_bounds__(AT_THREADS, DP == 256 ? 2 : 3) k_kv_span_cc(const __grid_constant__ SpanArgs g) {
    extern __shared__ __align__(16) float kv_smem[];
    using Hd = Held<T>;
    const AttendArgs& a = g.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    ptx::grid_dep_launch();
    const Piece x = piece_of(a, blockIdx.x, warp);
    const SidePlan& sp = a.o;
    const KvSide& s = a.c.own;
    const int D = a.c.D;
    float* qs = kv_smem + warp / sp.wk * (KR_ROWS * DP);
    const int wk = warp % sp.wk;
    float* ps = kv_smem + CcSmem<DP, JOIN>::P_OFF / 4 + warp * (32 * KR_ROWS);
    if (wk == 0) {
        for (int e0 = lane; e0 < KR_ROWS * (DP / 4); e0 += 4 * 32) {
            float4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = e0 + 32 * i, r = x.t.r0 + e / (DP / 4), d = 4 * (e % (DP / 4));
                v[i] = r < x.t.R && d < D ? *(const float4*)(static_cast<const float*>(a.c.q) + row_query(a.c, x.t, r) + d)
                                          : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) *(float4*)(qs + 4 * (e0 + 32 * i)) = v[i];
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
    constexpr int NI = (DP + 127) / 128, VL = 4 / NI;   // values on their way
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
        float2 p2[KR_ROWS];
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) p2[r] = make_float2(0.f, 0.f);
        const bool live = span_sees(g.s, key, lim, first);   // by some row of the tile
        const T* kp = kbase + (live ? key * s.rs : 0);
        float ks = 1.f, vs = 1.f;
        if (HELD8 && live) {
            ks = kv8_scale(g.s.ks[scales + (key >> g.s.n_log2)]);
            vs = kv8_scale(g.s.vs[scales + (key >> g.s.n_log2)]);
        }
        // Values of VL keys, those of the next ones on their way while these are used, the first ones during the scores.
        typename Hd::Four next[VL][NI];
        auto load = [&](int t0) {
#pragma unroll
            for (int t = 0; t < VL; ++t)
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int d = 4 * lane + 128 * i;
                    next[t][i] = d < D && span_sees(g.s, key0 + t0 + t, lim, first) ? Hd::four(vbase + (key0 + t0 + t) * s.rs + d) : Hd::none();
                }
        };
        load(0);
        if (live) {
            typename Hd::Run k, k2;
            Hd::load(k, kp, D);
            for (int d0 = 0; d0 < D; d0 += Hd::RUN) {
                if (d0 + Hd::RUN < D) Hd::load(k2, kp + d0 + Hd::RUN, D - d0 - Hd::RUN);
#pragma unroll
                for (int i = 0; i < Hd::RUN / 4; ++i) {
                    if (d0 + 4 * i >= D) break;
                    float4 y = Hd::part(k, i);
                    // (a key by itself: its products with a query may pass fp32's range where those with it do not)
                    if (HELD8) y = make_float4(y.x * ks, y.y * ks, y.z * ks, y.w * ks);
#pragma unroll
                    for (int r = 0; r < KR_ROWS; ++r) {
                        const float4 q = *(const float4*)(qs + r * DP + d0 + 4 * i);
                        // (to D = 128 pairs would take registers that the loads ahead need)
                        if constexpr (DP == 256) p2[r] = fma2(make_float2(q.x, q.y), make_float2(y.x, y.y), fma2(make_float2(q.z, q.w), make_float2(y.z, y.w), p2[r]));
                        else p2[r].x = fmaf(q.x, y.x, fmaf(q.y, y.y, fmaf(q.z, y.z, fmaf(q.w, y.w, p2[r].x))));
                    }
                }
                k = k2;
            }
        }
        __syncwarp();   // (and the last block's probabilities have been read)
        float p[KR_ROWS];
        bool cut = false;   // some row does not see all of the block's keys
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) {
            const bool in = span_sees(g.s, key, n[r], span_first(g.s, n[r]));
            cut = cut || !in;
            const float sc = in ? p2[r].x + p2[r].y : -INFINITY;
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
        cut = __any_sync(0xffffffffu, cut);
        *(float4*)(ps + 8 * lane) = make_float4(p[0], p[1], p[2], p[3]);
        *(float4*)(ps + 8 * lane + 4) = make_float4(p[4], p[5], p[6], p[7]);
        __syncwarp();
        for (int t0 = 0; t0 < 32 && key0 + t0 < lim; t0 += VL) {
            float4 v[VL][NI];
#pragma unroll
            for (int t = 0; t < VL; ++t)
#pragma unroll
                for (int i = 0; i < NI; ++i) v[t][i] = Hd::value(next[t][i]);
            if (t0 + VL < 32) load(t0 + VL);
            if constexpr (HELD8) {
#pragma unroll
                for (int t = 0; t < VL; ++t) {
                    const float by = __shfl_sync(0xffffffffu, vs, t0 + t);
#pragma unroll
                    for (int i = 0; i < NI; ++i) v[t][i] = make_float4(v[t][i].x * by, v[t][i].y * by, v[t][i].z * by, v[t][i].w * by);
                }
            }
            // A hidden value is multiplied by a probability of zero where it is finite, else by nothing.
            bool bad = false;
            if (cut) {
                float z = 0.f;
#pragma unroll
                for (int t = 0; t < VL; ++t)
#pragma unroll
                    for (int i = 0; i < NI; ++i) z = fmaf(v[t][i].x, 0.f, fmaf(v[t][i].y, 0.f, fmaf(v[t][i].z, 0.f, fmaf(v[t][i].w, 0.f, z))));
                bad = __any_sync(0xffffffffu, !(z == 0.f));
            }
            // (Apart from each other: with the test in one path, 4 requests of 40 tokens over 2000 keys of 64 took 55 us for 46.)
            auto add = [&](auto check) {
#pragma unroll
                for (int t = 0; t < VL; ++t) {
                    const float4 wa = *(const float4*)(ps + 8 * (t0 + t)), wb = *(const float4*)(ps + 8 * (t0 + t) + 4);
                    const float w[KR_ROWS] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
#pragma unroll
                    for (int r = 0; r < KR_ROWS; ++r) {
                        if (check.value && !span_sees(g.s, key0 + t0 + t, n[r], span_first(g.s, n[r]))) continue;
#pragma unroll
                        for (int i = 0; i < NI; ++i) {
                            const float2 xy = fma2(make_float2(w[r], w[r]), make_float2(v[t][i].x, v[t][i].y), make_float2(o[r][i].x, o[r][i].y));
                            const float2 zw = fma2(make_float2(w[r], w[r]), make_float2(v[t][i].z, v[t][i].w), make_float2(o[r][i].z, o[r][i].w));
                            o[r][i] = make_float4(xy.x, xy.y, zw.x, zw.y);
                        }
                    }
                }
            };
            if (bad) add(std::true_type{});
            else add(std::false_type{});
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
    if constexpr (JOIN) {
        __syncthreads();
        join_cluster<DP, float, AT_WARPS, MergeSmem<DP>::WARP_FLOATS * 4>(a, x, sp.splits, reinterpret_cast<uint8_t*>(kv_smem), warp, lane);
    } else {
        merge_and_write<DP, float>(a, x, sp, kv_smem, warp, lane);
    }
}

// bf16 queries. A warp works alone: it takes pieces (8 query rows over a range of the blocks that they see) in turn and streams
// their blocks of keys, 16 KB with their values (8 of codes), through two stages of shared memory of its own by 16-byte asynchronous
// copies, the next piece's first blocks and query rows behind this one's last; rows behind the piece's largest count, or before
// its windows and behind the first `sink`, arrive as zeros and are not read. Keys are the 16 rows of mma.sync m16n8k16 and query rows its 8 columns; the values' product runs over keys
// with d as its rows, the probabilities turned from one's result into the other's operand by 8 x 8 transposes.
//
// In 8 bits the codes become fp16 numbers on their way from shared memory into the fragments, two by one instruction: e4m3 is a
// subset of fp16. What a lane reads as 32 bits of a key are four elements of d, taken as the fragment's two pairs (the
// queries' are taken alike); of the values, by a transposing load, two elements of d of two keys, whose bytes one
// permutation brings together by keys, so that the fragment's rows g and g + 8 are elements 2 g and 2 g + 1. A block's scale
// multiplies its scores, and its probabilities before the second product: relative to the largest scale 2^e that the row
// has seen, p 2^(e_j - e) 2^7 is at most 2^15, and as an fp16 number is off by 2^-11 of itself or 2^-32 times 2^(e - e_j) (fp16's least
// step, 2^-24). Probabilities of bf16 caches enter as two bf16 terms (the rounded value and what the rounding left).
//
// A call of few tiles, which is waited for, takes one launch (JOIN): a cluster of blocks has a tile, each of its warps a part, and
// the parts are joined through the blocks' shared memories in place of the workspace and a second kernel.
template <int DP, bool Q8>
struct SrSmem {
    // A block's keys and values. Codes take twice the instructions a byte, and what bounds them is a warp's latency: smaller blocks, more
    // warps. (64 requests over 16384 rows of one KV head of 256: 129 us with five warps an SM, 16 KB each twice.)
    static constexpr int STAGE = Q8 ? 8192 : 16384;
    static constexpr int ROW = Q8 ? DP : 2 * DP;         // bytes of a key
    static constexpr int KEYS = STAGE / 2 / ROW;         // keys of a block
    static constexpr int HALF = STAGE / 2;
    static constexpr int QBYTES = KR_ROWS * DP * 2;
    static constexpr int Q_OFF = 2 * STAGE;
    static constexpr int SEEN_OFF = Q_OFF + 2 * QBYTES;  // [AHEAD][8] counts of the pieces in hand
    static constexpr int AHEAD = 4;
    static constexpr int BYTES = SEEN_OFF + AHEAD * KR_ROWS * 4;
    static constexpr int ALONE = Q8 ? (DP == 256 ? 8 : DP == 128 ? 10 : 11) : DP == 256 ? 5 : 6;   // blocks of an SM
    static constexpr int REGS = 65536 / 32 / ALONE / 8 * 8 < 255 ? 65536 / 32 / ALONE / 8 * 8 : 255;
    // JOIN: warps of a block, each with all of this for itself; in 8 bits by the registers, else as many as fit (one token over windows of 1024
    // rows of 256 8.1 us; with four warps 9.0).
    static constexpr int TEAM = Q8 ? 8 : DP == 256 ? 5 : 6;
    static constexpr int JOIN_BYTES = JoinSmem<DP, __nv_bfloat16, TEAM, BYTES>::BYTES;
    static_assert(BYTES % 128 == 0 && MergeSmem<DP>::WARP_FLOATS * 4 <= 2 * STAGE, "a warp's rows fit its stages");
};
__device__ __forceinline__ void sr_ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void sr_ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
// D += A B as kr_mma, fp16 operands.
__device__ __forceinline__ void sr_mma_half(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                            uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t sr_half2(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

constexpr int SR_NONE = -4096;   // no scale seen yet

template <int DP, bool Q8, bool JOIN>
__global__ void __maxnreg__((JOIN ? 248 : SrSmem<DP, Q8>::REGS)) k_kv_span_rows(const __grid_constant__ SpanArgs g_) {
    using L = SrSmem<DP, Q8>;
    using T = typename std::conditional<Q8, uint8_t, __nv_bfloat16>::type;
    extern __shared__ __align__(128) uint8_t sr_block[];
    const int warp = JOIN ? (int)threadIdx.x >> 5 : 0, lane = JOIN ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    uint8_t* const sr_smem = sr_block + warp * L::BYTES;   // this warp's own
    const AttendArgs& a = g_.a;
    const KvSpan& sn = g_.s;
    constexpr int MT = L::KEYS / 16;   // 16-key tiles of a block
    constexpr int ND = DP / 16;
    constexpr int EPC = Q8 ? 16 : 8;   // elements of a 16-byte chunk
    constexpr int CH = DP / EPC;       // chunks of a row; chunk c of row r lies at c ^ turn(r)
    constexpr int RPI = 32 / CH;       // rows one instruction of the warp copies
    constexpr int QCH = DP / 8, QRPI = 32 / QCH;
    const int g = lane >> 2, j = lane & 3;
    const uint32_t sm = ptx::smem_u32(sr_smem);
    int* const counts = (int*)(sr_smem + L::SEEN_OFF);
    ptx::grid_dep_launch();
    const uint32_t pieces = (uint32_t)a.o.blocks;
    const uint32_t mine0 = JOIN ? blockIdx.x * L::TEAM + warp : blockIdx.x, step = JOIN ? pieces : gridDim.x;   // its first piece; to the next
    const KvSide& s = a.c.own;
    const int D = a.c.D, mych = lane % CH, myrow = lane / CH;
    const bool dlive = EPC * mych < D;
    const float slack = 8.f / a.c2;
    auto turn = [](int r) { return CH == 4 ? (r >> 1) & 3 : r & 7; };

    // ---- what is to be copied: pieces opened in order, block by block
    uint32_t f_piece = mine0;
    int f_seq = 0, f_full = 0, f_blk = 0, f_end = 0, f_lim = 0, f_first = 0;
    SpanBlocks<L::KEYS> f_blocks(sn, 0, 0);
    const T *f_k = nullptr, *f_v = nullptr;   // this lane's chunk of the open piece's row 0
    const uint8_t* f_s = nullptr;             // scales of the open piece's keys (lanes below 16) or values
    int s_new = 0, s_old = 0;                 // scales of the last block asked for, and the one before: tile lane % 16
    int ahead = 0;                            // this lane's row's count of the next piece (lanes 0-7)
    auto peek = [&]() {
        ahead = 0;
        if (f_piece < pieces) {
            const Piece x = piece_of(a, f_piece, 0);
            if (lane < KR_ROWS) ahead = row_seen(a.c, false, x.cache, x.t, x.t.r0 + lane);
        }
    };
    int issued = 0, used = 0;
    int seq = 0, full = 0;
    auto produce = [&]() {
        while (f_blk >= f_end) {
            if (f_piece >= pieces || f_seq - seq >= L::AHEAD) return false;
            const Piece x = piece_of(a, f_piece, 0);
            if (lane < KR_ROWS) counts[(f_seq & (L::AHEAD - 1)) * KR_ROWS + lane] = ahead;
            f_lim = __reduce_max_sync(0xffffffffu, lane < KR_ROWS ? ahead : 0);
            f_first = __reduce_min_sync(0xffffffffu, lane < KR_ROWS && ahead > 0 ? span_first(sn, ahead) : 0x7fffffff);
            f_blocks = SpanBlocks<L::KEYS>(sn, f_lim, f_first);
            f_blk = (int)((long long)f_blocks.count * x.split / a.o.splits);
            f_end = (int)((long long)f_blocks.count * (x.split + 1) / a.o.splits);
            if (f_blk < f_end) {
                const long long base = x.cache * s.cs + x.kvh * s.hs + (dlive ? EPC * mych : 0);
                f_k = static_cast<const T*>(s.k) + base;
                f_v = static_cast<const T*>(s.v) + base;
                if (Q8) f_s = (lane < 16 ? sn.ks : sn.vs) + ((long long)x.cache * a.c.K + x.kvh) * sn.nblk;
                // The query rows travel with the first block. (Two pieces' fit: with two blocks in hand, the piece with
                // blocks before the last one is through.)
#pragma unroll
                for (int i = 0; i < KR_ROWS / QRPI; ++i) {
                    const int rr = i * QRPI + lane / QCH, r = x.t.r0 + rr, ch = lane % QCH;
                    const bool in = 8 * ch < D && r < x.t.R;
                    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.c.q) + (in ? row_query(a.c, x.t, r) + 8 * ch : 0);
                    ptx::cp_async_16(sm + L::Q_OFF + (f_full & 1) * L::QBYTES + rr * (DP * 2) + ((ch ^ (rr & 7)) << 4), q, in);
                }
                ++f_full;
            }
            ++f_seq;
            f_piece += step;
            peek();
        }
        const uint32_t dst = sm + (issued & 1) * L::STAGE;
        const int key0 = f_blocks.row(f_blk);
        const T *k = f_k + (long long)(key0 + myrow) * s.rs, *v = f_v + (long long)(key0 + myrow) * s.rs;
        if (key0 + L::KEYS <= f_lim && (key0 >= f_first || key0 + L::KEYS <= sn.sink)) {   // all seen, as most are
#pragma unroll
            for (int i = 0; i < L::KEYS / RPI; ++i) {
                const int rr = i * RPI + myrow;
                const uint32_t at = rr * L::ROW + ((mych ^ turn(rr)) << 4);
                ptx::cp_async_16(dst + at, k, dlive);
                ptx::cp_async_16(dst + L::HALF + at, v, dlive);
                k += RPI * s.rs;
                v += RPI * s.rs;
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < L::KEYS / RPI; ++i) {
                const int rr = i * RPI + myrow;
                const bool in = dlive && span_sees(sn, key0 + rr, f_lim, f_first);
                const uint32_t at = rr * L::ROW + ((mych ^ turn(rr)) << 4);
                ptx::cp_async_16(dst + at, in ? k : f_k, in);
                ptx::cp_async_16(dst + L::HALF + at, in ? v : f_v, in);
                k += RPI * s.rs;
                v += RPI * s.rs;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (Q8) {
            s_old = s_new;
            const int tile = key0 + 16 * (lane & 15);
            // (a tile that no row sees has no scale)
            const bool in = (lane & 15) < MT && tile < f_lim && (tile < sn.sink || tile + 16 > f_first);
            s_new = in ? (int)f_s[tile >> sn.n_log2] : -1;
        }
        ++issued;
        ++f_blk;
        return true;
    };

    peek();
    if (produce()) produce();
    for (uint32_t piece = mine0; piece < pieces; piece += step, ++seq) {
        const Piece x = piece_of(a, piece, 0);
        if (f_seq <= seq) produce();
        __syncwarp();
        // What the lane's rows 2 j, 2 j + 1 see, and the tile's rows together.
        const int n0 = counts[(seq & (L::AHEAD - 1)) * KR_ROWS + 2 * j], n1 = counts[(seq & (L::AHEAD - 1)) * KR_ROWS + 2 * j + 1];
        const int w0 = span_first(sn, n0), w1 = span_first(sn, n1);
        const int rj = x.t.r0 + 2 * j;
        const bool in0 = rj < x.t.R, in1 = rj + 1 < x.t.R;
        int lim = max(n0, n1), low = min(in0 ? n0 : 0x7fffffff, in1 ? n1 : 0x7fffffff);     // counts: most, least
        int first = min(n0 > 0 ? w0 : 0x7fffffff, n1 > 0 ? w1 : 0x7fffffff), late = max(w0, w1);   // first rows: least, most
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            lim = max(lim, __shfl_xor_sync(0xffffffffu, lim, o));
            low = min(low, __shfl_xor_sync(0xffffffffu, low, o));
            first = min(first, __shfl_xor_sync(0xffffffffu, first, o));
            late = max(late, __shfl_xor_sync(0xffffffffu, late, o));
        }
        const SpanBlocks<L::KEYS> blocks(sn, lim, first);
        const int b0 = (int)((long long)blocks.count * x.split / a.o.splits), b1 = (int)((long long)blocks.count * (x.split + 1) / a.o.splits);
        uint32_t qf[ND][2];
        float qs0 = 1.f, qs1 = 1.f;    // Q8: what the rows' queries were divided by
        float o[ND][4];
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        int v0 = SR_NONE, v1 = SR_NONE;   // Q8: the largest scale of values that the rows have seen
        for (int blk = b0; blk < b1; ++blk) {
            const int key0 = blocks.row(blk);
            if (issued == used) produce();
            int scale = 0;
            if (issued - used > 1) {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                if (Q8) scale = s_old;
            } else {
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                if (Q8) scale = s_new;
            }
            __syncwarp();
            const uint32_t ks = sm + (used & 1) * L::STAGE, vs = ks + L::HALF;
            if (blk == b0) {
                const uint32_t qb = L::Q_OFF + (full++ & 1) * L::QBYTES;
                if constexpr (Q8) {
                    const uint8_t* row = sr_smem + qb + g * (DP * 2) + (j & 1) * 8;
                    auto at = [&](int i) { return *(const uint2*)(row + (((2 * i + (j >> 1)) ^ g) << 4)); };
                    float top = 0.f;
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        const uint2 u = at(i);
                        const uint32_t w[2] = {u.x & 0x7fff7fffu, u.y & 0x7fff7fffu};
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float lo = __uint_as_float(w[e] << 16), hi = __uint_as_float(w[e] & 0xffff0000u);
                            top = fmaxf(top, lo < INFINITY ? lo : 0.f);
                            top = fmaxf(top, hi < INFINITY ? hi : 0.f);
                        }
                    }
#pragma unroll
                    for (int e = 1; e < 4; e <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, e));
                    // The largest to 2 .. 4: elements keep bf16's bits down to 2^-14 of it.
                    const int E = max((int)(__float_as_uint(top) >> 23), 2);
                    const float f = kv8_pow2(255 - E), q = kv8_pow2(E - 1);
                    qs0 = __shfl_sync(0xffffffffu, q, 8 * j);
                    qs1 = __shfl_sync(0xffffffffu, q, 8 * j + 4);
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        const uint2 u = at(i);
                        qf[i][0] = sr_half2(__uint_as_float(u.x << 16) * f, __uint_as_float(u.x & 0xffff0000u) * f);
                        qf[i][1] = sr_half2(__uint_as_float(u.y << 16) * f, __uint_as_float(u.y & 0xffff0000u) * f);
                    }
                } else {
                    const uint32_t qa = sm + qb + (lane & 7) * (DP * 2);
#pragma unroll
                    for (int i = 0; i < ND; i += 2) {
                        uint32_t f[4];
                        sr_ldsm4(f, qa + (((2 * i + (lane >> 3)) ^ (lane & 7)) << 4));
                        qf[i][0] = f[0];
                        qf[i][1] = f[1];
                        qf[i + 1][0] = f[2];
                        qf[i + 1][1] = f[3];
                    }
                }
            }
            // Four chains of products whatever the shape: one of D / 16 steps would be its latency.
            constexpr int NCH = MT >= 4 ? 1 : 4 / MT;
            float part[NCH][MT][4];
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[c][t][e] = 0.f;
            const int kr = (lane & 7) + (lane & 8);   // key of this lane's matrix row; its chunk is 2 i + lane / 16
            if constexpr (Q8) {
#pragma unroll
                for (int i = 0; i < ND; i += 2)
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        uint32_t f[4];
                        sr_ldsm4(f, ks + (16 * t + kr) * L::ROW + (((i + (lane >> 4)) ^ turn(kr)) << 4));
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            sr_mma_half(part[(i + c) % NCH][t], kv8_half2(f[2 * c]), kv8_half2(f[2 * c + 1]), kv8_half2(f[2 * c] >> 16),
                                        kv8_half2(f[2 * c + 1] >> 16), qf[i + c][0], qf[i + c][1]);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < ND; ++i)
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        uint32_t f[4];
                        sr_ldsm4(f, ks + (16 * t + kr) * L::ROW + (((2 * i + (lane >> 4)) ^ turn(kr)) << 4));
                        kr_mma(part[i % NCH][t], f[0], f[1], f[2], f[3], qf[i][0], qf[i][1]);
                    }
            }
            float sc[MT][4];
            const float mine = Q8 ? kv8_scale((uint32_t)max(scale, 0)) : 1.f;   // of tile lane % 16: keys below lane 16, values from there
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const float by = Q8 ? __shfl_sync(0xffffffffu, mine, t) : 1.f;
                // A row's factor below 1 first: the product with the other may pass fp32's range where the score does not.
                const float a0 = qs0 < 1.f ? qs0 : by, b0 = qs0 < 1.f ? by : qs0, a1 = qs1 < 1.f ? qs1 : by, b1 = qs1 < 1.f ? by : qs1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sc[t][e] = part[0][t][e];
#pragma unroll
                    for (int c = 1; c < NCH; ++c) sc[t][e] += part[c][t][e];
                    if (Q8) sc[t][e] = sc[t][e] * (e & 1 ? a1 : a0) * (e & 1 ? b1 : b0);
                }
            }
            // Keys g, g + 8 of each tile, rows 2 j, 2 j + 1; hidden scores are replaced, whatever they hold.
            const bool cut = low < key0 + L::KEYS || (key0 < late && key0 + L::KEYS > sn.sink);   // the same for the warp
            if (cut) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = key0 + 16 * t + g + 8 * e;
                        if (!span_sees(sn, key, n0, w0)) sc[t][2 * e] = -INFINITY;
                        if (!span_sees(sn, key, n1, w1)) sc[t][2 * e + 1] = -INFINITY;
                    }
            }
            float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    x0 = fmaxf(x0, sc[t][2 * e]);
                    x1 = fmaxf(x1, sc[t][2 * e + 1]);
                }
            float a0 = 1.f, a1 = 1.f;      // what the outputs so far are multiplied by
            bool moved = false;            // (of the warp)
            // The maximum moves only when a score passes it by more than 8 in log2 units (probabilities stay below 2^8):
            // most blocks do not, and need no maximum over the keys' lanes.
            if (__any_sync(0xffffffffu, x0 > m0 + slack || x1 > m1 + slack)) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, d));
                    x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, d));
                }
                const float y0 = fmaxf(m0, x0), y1 = fmaxf(m1, x1);
                a0 = m0 == -INFINITY ? 0.f : kr_ex2((m0 - y0) * a.c2);
                a1 = m1 == -INFINITY ? 0.f : kr_ex2((m1 - y1) * a.c2);
                m0 = y0;
                m1 = y1;
                l0 *= a0;
                l1 *= a1;
                moved = true;
            }
            // Likewise the largest scale of the values: outputs are in units of it.
            if constexpr (Q8) {
                const int top = __reduce_max_sync(0xffffffffu, lane >= 16 && scale < 255 ? scale : -1);
                if (__any_sync(0xffffffffu, top > v0 || top > v1)) {
                    int t0 = v0, t1 = v1;
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        const int e = __shfl_sync(0xffffffffu, scale, 16 + t), tile = key0 + 16 * t;
                        if (e >= 0 && e < 255) {
                            if (tile < n0 && (tile < sn.sink || tile + 16 > w0)) t0 = max(t0, max(e, 1));
                            if (tile < n1 && (tile < sn.sink || tile + 16 > w1)) t1 = max(t1, max(e, 1));
                        }
                    }
                    a0 *= kv8_pow2(127 + v0 - t0);
                    a1 *= kv8_pow2(127 + v1 - t1);
                    v0 = t0;
                    v1 = t1;
                    moved = true;
                }
            }
            if (moved) {
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
            for (int t = 0; t < MT; ++t) {
                float by0 = 1.f, by1 = 1.f;
                if (Q8) {
                    const int e = __shfl_sync(0xffffffffu, scale, 16 + t);
                    by0 = e == 255 ? NAN : kv8_pow2(min(134 + e - v0, 254));
                    by1 = e == 255 ? NAN : kv8_pow2(min(134 + e - v1, 254));
                    if (e < 0) by0 = by1 = 1.f;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float p0 = kr_ex2((sc[t][2 * e] - f0) * a.c2), p1 = kr_ex2((sc[t][2 * e + 1] - f1) * a.c2);
                    l0 += p0;
                    l1 += p1;
                    if constexpr (Q8) {
                        ph[t][e] = kr_transpose(sr_half2(p0 * by0, p1 * by1));
                    } else {
                        const uint32_t h = kr_pack(p0, p1);
                        const uint32_t r = kr_pack(p0 - __uint_as_float(h << 16), p1 - __uint_as_float(h & 0xffff0000u));
                        ph[t][e] = kr_transpose(h);
                        pe[t][e] = kr_transpose(r);
                    }
                }
            }
            if constexpr (Q8) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < ND; i += 2) {
                        uint32_t f[4];
                        sr_ldsm4_t(f, vs + (16 * t + kr) * L::ROW + (((i + (lane >> 4)) ^ turn(kr)) << 4));
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const uint32_t lo = __byte_perm(f[2 * c], 0, 0x3120), hi = __byte_perm(f[2 * c + 1], 0, 0x3120);
                            const uint32_t u0 = kv8_half2(lo), u1 = kv8_half2(lo >> 16), u2 = kv8_half2(hi), u3 = kv8_half2(hi >> 16);
                            sr_mma_half(o[i + c], u0, u1, u2, u3, ph[t][0], ph[t][1]);
                        }
                    }
            } else {
                const int vr = (lane & 7) + ((lane >> 4) << 3);   // key of this lane's matrix row; its chunk is 2 i + bit 3
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        uint32_t f[4];
                        sr_ldsm4_t(f, vs + (16 * t + vr) * L::ROW + (((2 * i + ((lane >> 3) & 1)) ^ turn(vr)) << 4));
                        kr_mma(o[i], f[0], f[1], f[2], f[3], ph[t][0], ph[t][1]);
                        kr_mma(o[i], f[0], f[1], f[2], f[3], pe[t][0], pe[t][1]);
                    }
            }
            __syncwarp();   // every lane has read the stage
            ++used;
            produce();
        }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        if (Q8) {
            const float u0 = v0 == SR_NONE ? 0.f : kv8_scale((uint32_t)v0), u1 = v1 == SR_NONE ? 0.f : kv8_scale((uint32_t)v1);
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                o[i][0] = o[i][0] * 0x1p-7f * u0;
                o[i][1] = o[i][1] * 0x1p-7f * u1;
                o[i][2] = o[i][2] * 0x1p-7f * u0;
                o[i][3] = o[i][3] * 0x1p-7f * u1;
            }
        }
        // Element e (0, 1: rows 2 j and 2 j + 1; 2, 3 likewise) of fragment i.
        auto elem = [&](int i, int half) { return Q8 ? 16 * i + 2 * g + half : 16 * i + g + 8 * half; };
        // An infinite value times what the rounding left of its probability (0, or of the other sign) is NaN, and so is 0 times an
        // infinity or NaN that only another row of the tile sees. Rows whose sum is finite and outputs are not are formed
        // again, key by key in fp32, each over its own keys.
        float z0 = 0.f, z1 = 0.f;   // 0 as long as all are finite
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            z0 = fmaf(o[i][0], 0.f, fmaf(o[i][2], 0.f, z0));
            z1 = fmaf(o[i][1], 0.f, fmaf(o[i][3], 0.f, z1));
        }
        uint32_t again = __reduce_or_sync(0xffffffffu, (in0 && l0 < INFINITY && !(z0 == 0.f) ? 1u << (2 * j) : 0u) |
                                                           (in1 && l1 < INFINITY && !(z1 == 0.f) ? 2u << (2 * j) : 0u));
        for (; again; again &= again - 1) {
            const int r = __ffs(again) - 1;
            const int n = __shfl_sync(0xffffffffu, (r & 1) ? n1 : n0, r >> 1);
            float m = __shfl_sync(0xffffffffu, (r & 1) ? m1 : m0, r >> 1);
            if (m == -INFINITY) m = 0.f;
            constexpr int NL = DP / 32;   // lane's elements of a row: lane + 32 i
            const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.c.q) + row_query(a.c, x.t, x.t.r0 + r);
            const long long base = x.cache * s.cs + x.kvh * s.hs;
            const long long sb = ((long long)x.cache * a.c.K + x.kvh) * sn.nblk;
            auto value = [](T u) {
                if constexpr (Q8) return __half2float(__ushort_as_half((unsigned short)kv8_half2(u)));
                else return __bfloat162float(u);
            };
            float qr[NL], sum[NL];
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                qr[i] = lane + 32 * i < D ? __bfloat162float(q[lane + 32 * i]) : 0.f;
                sum[i] = 0.f;
            }
#pragma unroll 1
            for (int e = b0 * L::KEYS; e < b1 * L::KEYS; ++e) {
                const int key = blocks.row(e / L::KEYS) + e % L::KEYS;
                if (!span_sees(sn, key, n, span_first(sn, n))) continue;
                const T *k = static_cast<const T*>(s.k) + base + key * s.rs, *v = static_cast<const T*>(s.v) + base + key * s.rs;
                float dot = 0.f, ksc = 1.f, vsc = 1.f;
                if (Q8) {
                    ksc = kv8_scale(sn.ks[sb + (key >> sn.n_log2)]);
                    vsc = kv8_scale(sn.vs[sb + (key >> sn.n_log2)]);
                }
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    if (lane + 32 * i < D) dot = fmaf(qr[i], value(k[lane + 32 * i]) * ksc, dot);
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
                const float pr = kr_ex2((dot - m) * a.c2);
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    if (lane + 32 * i < D) sum[i] = fmaf(pr, value(v[lane + 32 * i]) * vsc, sum[i]);
            }
            // Back to the fragments, through the lanes that hold the elements.
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                const float y0 = __shfl_sync(0xffffffffu, sum[i >> 1], elem(i, 0) & 31), y1 = __shfl_sync(0xffffffffu, sum[i >> 1], elem(i, 1) & 31);
                if (r == 2 * j) o[i][0] = y0, o[i][2] = y1;
                if (r == 2 * j + 1) o[i][1] = y0, o[i][3] = y1;
            }
        }
        if constexpr (JOIN) {
            // The warp's rows go where its stages were, whose copies have all been read.
            constexpr int LD = MergeSmem<DP>::LD;
            float* f = reinterpret_cast<float*>(sr_smem);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    f[2 * j * LD + elem(i, e)] = o[i][2 * e];
                    f[(2 * j + 1) * LD + elem(i, e)] = o[i][2 * e + 1];
                }
            if (g == 0) {
                *(float2*)(f + KR_ROWS * LD + 4 * j) = make_float2(m0, l0);
                *(float2*)(f + KR_ROWS * LD + 4 * j + 2) = make_float2(m1, l1);
            }
            __syncthreads();
            join_cluster<DP, __nv_bfloat16, L::TEAM, L::BYTES>(a, x, a.o.splits / L::TEAM, sr_block, warp, lane);
            return;
        }
        const long long row0 = in0 ? row_index(a.c, x.t, rj) : 0, row1 = in1 ? row_index(a.c, x.t, rj + 1) : 0;
        if (a.out) {
            const float inv0 = inverse_sum(l0), inv1 = inverse_sum(l1);
            __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(a.out);
            if constexpr (Q8) {
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    if (16 * i >= D) continue;
                    if (in0) *(uint32_t*)(out + row0 * D + elem(i, 0)) = kr_pack(o[i][0] * inv0, o[i][2] * inv0);
                    if (in1) *(uint32_t*)(out + row1 * D + elem(i, 0)) = kr_pack(o[i][1] * inv1, o[i][3] * inv1);
                }
            } else {
                // Lanes g and g + 1 exchange halves, so that the even one has a pair of row 2 j and the odd one of row 2 j + 1.
                const bool even = (g & 1) == 0;
                __nv_bfloat16* dst = out + (even ? row0 : row1) * D + (g & ~1);
#pragma unroll
                for (int i = 0; i < ND; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float u = o[i][2 * e] * inv0, v = o[i][2 * e + 1] * inv1;
                        const float w = __shfl_xor_sync(0xffffffffu, even ? v : u, 4);
                        if ((even ? in0 : in1) && 16 * i + 8 * e < D)
                            *(uint32_t*)(dst + 16 * i + 8 * e) = even ? kr_pack(u, w) : kr_pack(w, v);
                    }
            }
            if (g == 0 && a.lse) {
                if (in0) a.lse[row0] = log_sum(m0, l0, a.c.scale);
                if (in1) a.lse[row1] = log_sum(m1, l1, a.c.scale);
            }
        } else {
            const long long at0 = x.part * a.rows + row0, at1 = x.part * a.rows + row1;
            if (g == 0 && in0) a.pml[row0 * a.parts + x.part] = make_float2(m0, l0);
            if (g == 0 && in1) a.pml[row1 * a.parts + x.part] = make_float2(m1, l1);
            const bool u0 = in0 && l0 != 0.f, u1 = in1 && l1 != 0.f;
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                if constexpr (Q8) {
                    if (16 * i >= D) continue;
                    if (u0) *(float2*)(a.po + at0 * D + elem(i, 0)) = make_float2(o[i][0], o[i][2]);
                    if (u1) *(float2*)(a.po + at1 * D + elem(i, 0)) = make_float2(o[i][1], o[i][3]);
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (16 * i + 8 * e >= D) continue;
                        if (u0) a.po[at0 * D + elem(i, e)] = o[i][2 * e];
                        if (u1) a.po[at1 * D + elem(i, e)] = o[i][2 * e + 1];
                    }
                }
            }
        }
    }
}

// The kernels of a handle and their shared memory: on its own, and joined in clusters of blocks of `team` warps.
template <int DP>
struct SpanKernel {
    using Rows8 = SrSmem<DP, true>;
    using Rows = SrSmem<DP, false>;
    void (*alone)(SpanArgs), (*joined)(SpanArgs);
    int bytes, joined_bytes, keys, team;
    SpanKernel(const jpi_kv_handle* h, bool held8) {
        if (!h->bf16) {
            alone = held8 ? k_kv_span_cc<DP, Code8, false> : k_kv_span_cc<DP, float, false>;
            joined = held8 ? k_kv_span_cc<DP, Code8, true> : k_kv_span_cc<DP, float, true>;
            bytes = CcSmem<DP, false>::BYTES;
            joined_bytes = CcSmem<DP, true>::BYTES;
            keys = 32;
            team = AT_WARPS;
        } else {
            alone = held8 ? k_kv_span_rows<DP, true, false> : k_kv_span_rows<DP, false, false>;
            joined = held8 ? k_kv_span_rows<DP, true, true> : k_kv_span_rows<DP, false, true>;
            bytes = held8 ? Rows8::BYTES : Rows::BYTES;
            joined_bytes = held8 ? Rows8::JOIN_BYTES : Rows::JOIN_BYTES;
            keys = held8 ? Rows8::KEYS : Rows::KEYS;
            team = held8 ? Rows8::TEAM : Rows::TEAM;
        }
    }
};

// Rows of the cache that the tokens of a tile of 8 query rows see, with the ends of their blocks.
long long rows_span(const KvCall& c, const KvSpan& sn, int step) {
    const long long toks = std::min<long long>(c.tokens, (KR_ROWS + c.gq - 1) / c.gq + 1);
    return std::min<long long>(c.own.rows, (long long)sn.window + toks + std::min(sn.sink, c.own.rows) + 2 * step);
}

// How a call is dealt to blocks of `warps` warps, whose warps take `step` keys at a time: splits of the rows that a tile can see,
// up to `want` blocks in all while a warp keeps `least` keys; a call of few pieces, which is waited for, down to single steps as
// far as two blocks an SM go. The parts fit the workspace.
SidePlan plan_span(const jpi_kv_handle* h, const KvCall& c, const KvSpan& sn, int warps, int step, int least, long long want) {
    SidePlan s;
    const long long R = (long long)c.tokens * c.gq, rt = (R + KR_ROWS - 1) / KR_ROWS;
    while (s.wr < warps && s.wr < rt) s.wr *= 2;
    s.wk = warps / s.wr;
    s.tiles = (int)((rt + s.wr - 1) / s.wr);
    const long long rows = rows_span(c, sn, step);
    const long long blocks = (long long)c.batch * c.K * s.tiles, all = (long long)c.batch * c.tokens * c.H;
    const long long room = std::max(1ll, ws_rows(h) / all);
    const long long coarse = std::min(want / blocks, (rows + least * s.wk - 1) / (least * s.wk));
    const long long fine = std::min(2ll * h->num_sms / blocks, (rows + step * s.wk - 1) / (step * s.wk));
    s.splits = (int)std::max(1ll, std::min(std::max(coarse, fine), room));
    s.blocks = blocks * s.splits;
    s.by_splits = KvDiv((uint32_t)s.splits);
    s.by_tiles = KvDiv((uint32_t)s.tiles);
    return s;
}

// Blocks of the cluster that a small call's tile of query rows is dealt to: the most with which all clusters are resident together;
// 0: more tiles than fit one block each, or more blocks of keys for a warp than a second launch takes.
template <int DP>
int join_ranks(const jpi_kv_handle* h, const KvCall& c, const KvSpan& sn) {
    // (The fp32 kernel's blocks of one tile take the same time alone; with more than one they hold four tiles each there: 4 requests of 9
    // tokens over 300 keys of one KV head of 64 17 us, 14 joined, over 867 of 256 48 and 28.)
    if (!h->bf16 && (long long)c.tokens * c.gq <= KR_ROWS) return 0;
    const SpanKernel<DP> k(h, sn.ks != nullptr);
    const long long tiles = (long long)c.batch * c.K * (((long long)c.tokens * c.gq + KR_ROWS - 1) / KR_ROWS);
    const long long nb = (rows_span(c, sn, k.keys) + k.keys - 1) / k.keys;
    int n = 3;
    while (n >= 0 && tiles > h->span_clusters[sn.ks != nullptr][n]) --n;
    return n >= 0 && nb <= (long long)SR_JOIN_BLOCKS * k.team << n ? 1 << n : 0;
}

template <int DP>
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
    // Clusters first, wherever they have room for a call, also of many query rows: 128 rows over 300 keys of 256 9.8 us, on the 128-row tiles
    // 11.7, over 867 10.3 and 12.7; 16 heads of 64 at 64 tokens over 867 8.5 and 13.0. (JPI_KV_TILES=1 asks for the tiles.)
    if (const int ranks = h->tiles == 1 && h->bf16 ? 0 : join_ranks<DP>(h, c, sn)) {
        const SpanKernel<DP> k(h, sn.ks != nullptr);
        a.o.tiles = (int)(((long long)c.tokens * c.gq + KR_ROWS - 1) / KR_ROWS);
        a.o.wk = k.team;
        a.o.splits = h->bf16 ? ranks * k.team : ranks;   // (a block of the fp32 kernel is one split, whose keys its warps share)
        a.o.blocks = (long long)c.batch * c.K * a.o.tiles * a.o.splits;
        a.o.by_splits = KvDiv((uint32_t)a.o.splits);
        a.o.by_tiles = KvDiv((uint32_t)a.o.tiles);
        a.out = out;
        return kv_start_clusters(k.joined, dim3((unsigned)((long long)c.batch * c.K * a.o.tiles * ranks)), (unsigned)ranks, 32 * k.team,
                                 (size_t)k.joined_bytes, false, st, g);
    }
    bool joined;
    if (const int splits = kv_span_tiles_plan(h, c, sn, std::max(1ll, ws_rows(h) / a.rows), &joined)) {
        JPI_TRY(launch_kv_span_tiles(h, c, sn, splits, joined, a.po, a.pml, out, lse, st));
        return splits == 1 || joined ? JPI_OK : launch_kv_combine(h, c, splits, out, lse, st);
    }
    const SpanKernel<DP> k(h, sn.ks != nullptr);
    const long long most = (long long)(sn.ks ? SrSmem<DP, true>::ALONE : SrSmem<DP, false>::ALONE) * h->num_sms;   // resident warps of the row kernel
    if (h->bf16) a.o = plan_span(h, c, sn, 1, k.keys, 4 * k.keys, most);
    else a.o = plan_span(h, c, sn, AT_WARPS, 32, 32, 2ll * h->num_sms);
    a.p.splits = 0;
    a.parts = a.o.splits;
    if (a.o.blocks > 0x7fffffffll) {
        set_error("the call needs more than 2^31 blocks");
        return JPI_ERR_SHAPE;
    }
    if (a.parts == 1) a.out = out;
    const long long blocks = h->bf16 ? std::min(a.o.blocks, most) : a.o.blocks;   // (the row kernel's take pieces in turn)
    JPI_TRY(kv_start(k.alone, dim3((unsigned)blocks), h->bf16 ? 32 : AT_THREADS, (size_t)k.bytes, false, st, g));
    return a.parts == 1 ? JPI_OK : launch_kv_combine(h, c, a.parts, out, lse, st);
}

template <int DP>
jpi_status prepare_dim(jpi_kv_handle* h) {
    for (int held8 = 0; held8 < 2; ++held8) {
        const SpanKernel<DP> k(h, held8 != 0);
        JPI_CUDA_TRY(cudaFuncSetAttribute(k.alone, cudaFuncAttributeMaxDynamicSharedMemorySize, k.bytes));
        JPI_CUDA_TRY(cudaFuncSetAttribute(k.joined, cudaFuncAttributeMaxDynamicSharedMemorySize, k.joined_bytes));
        if (h->bf16)   // all of its loads go to shared memory
            JPI_CUDA_TRY(cudaFuncSetAttribute(k.alone, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
        for (int n = 0; n < 4; ++n)
            JPI_TRY(kv_resident_clusters(k.joined, 1u << n, 32 * k.team, (size_t)k.joined_bytes, &h->span_clusters[held8][n]));
    }
    return JPI_OK;
}

// The kernels' shared memory and the clusters that are resident together: by a handle's first call here, so that one that only appends, or
// attends over whole caches, does not load these kernels.
jpi_status kv_span_prepare(jpi_kv_handle* h) {
    JPI_TRY(kv_span_tiles_prepare(h));
    JPI_TRY(h->D <= 64 ? prepare_dim<64>(h) : h->D <= 128 ? prepare_dim<128>(h) : prepare_dim<256>(h));
    h->span_ready = true;
    return JPI_OK;
}

}  // namespace

jpi_status launch_kv_span(jpi_kv_handle* h, const KvCall& c, const KvSpan& s, void* out, float* lse, cudaStream_t st) {
    if (!h->span_ready) JPI_TRY(kv_span_prepare(h));
    return h->D <= 64 ? launch_dim<64>(h, c, s, out, lse, st)
                      : h->D <= 128 ? launch_dim<128>(h, c, s, out, lse, st) : launch_dim<256>(h, c, s, out, lse, st);
}

}  // namespace jpi
