// Heads held by groups of lanes: the norm of a head and its rotary coding in registers (kv_append_normed.cu, kv8_append.cu).
//
// A head of D elements is C = D / V chunks of 16 bytes. A group of G lanes (a power of two, at most a warp) holds it, two
// chunks a lane: in the half layout a pair's two chunks, so that a lane has both elements of each of its pairs and the
// rotation needs no exchange; else two neighbours. The sum of squares is a sum over the group by shuffles.
#pragma once

#include "kv_code.cuh"
#include "kv_pair.cuh"
#include "../ptx.h"

#include <algorithm>

namespace jpi {
namespace {

// What new tokens are coded by.
struct HeadArgs {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    const int* position;
    void* q_out;
    int H, K, D;                 // H = 0 without queries, K = 0 without keys
    int batch, tokens;
    KvDiv by_tokens;
    const uint64_t* turns;
    int dim;
    float m;
    bool norm;
    const float *q_weight, *k_weight;   // NULL: ones
    float eps, inv_d;            // 1 / D
    int lanes_log2;              // G
};

// Lanes of a group, log2.
inline int head_lanes_log2(int D, int V, int dim, int mode) {
    const int C = D / V, pairs = mode == RM_HALF ? dim / 2 / V : 0, units = pairs + (C - 2 * pairs + 1) / 2;
    int lg = 0;
    while ((1 << lg) < units) ++lg;
    return lg;
}

// A lane's two chunks (of C; beyond that: none) of a head.
template <typename E, int MODE>
struct HeadLane {
    static constexpr int V = Chunk<E>::V;
    int c[2];
    bool pair;     // the two hold the halves of V pairs
    bool live[2];
    __device__ __forceinline__ HeadLane(int u, int D, int dim) {
        const int pairs = MODE == RM_HALF ? dim / 2 / V : 0;
        pair = MODE == RM_HALF && u < pairs;
        c[0] = pair ? u : 2 * u;              // (2 pairs + 2 (u - pairs) = 2 u)
        c[1] = pair ? u + pairs : 2 * u + 1;
        live[0] = c[0] < D / V;
        live[1] = c[1] < D / V;
    }
    __device__ __forceinline__ void load(const E* head, bool in, uint4 (&raw)[2]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            raw[i] = in && live[i] ? *reinterpret_cast<const uint4*>(head + c[i] * V) : make_uint4(0, 0, 0, 0);
    }
};

__device__ __forceinline__ float group_sum(float x, int lanes_log2) {
    for (int i = 0; i < lanes_log2; ++i) x += __shfl_xor_sync(0xffffffffu, x, 1 << i);
    return x;
}

// 1 / sqrt(v): the hardware's approximation (2^-22) and one step of Newton's for the equation 1 / r^2 = v.
__device__ __forceinline__ float inverse_root(float v) {
    const float r = rsqrtf(v);
    return v < INFINITY ? r * fmaf(-0.5f * v * r, r, 1.5f) : r;
}

// Makes a head's elements x (those of one lane) x / sqrt(mean(x^2) + eps); returns the factors that did it, one after the other. Where
// that sum passes 1e38, and may pass fp32's range, the first is 2^-70 (the mean and eps are then 2^-140 of theirs), else it is 1. Every
// lane of the warp calls.
template <int N>
__device__ __forceinline__ float2 head_norm(float2 (&x)[N], float inv_d, float eps, int lanes_log2) {
    float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i) s2 = fma2(x[i], x[i], s2);
    const float v = fmaf(group_sum(s2.x + s2.y, lanes_log2), inv_d, eps);
    float2 r = make_float2(1.f, inverse_root(v));
    if (__any_sync(0xffffffffu, v > 1e38f)) {
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 y = make_float2(x[i].x * 0x1p-70f, x[i].y * 0x1p-70f);
            z = fmaf(y.x, y.x, fmaf(y.y, y.y, z));
            if (v > 1e38f) x[i] = y;
        }
        z = group_sum(z, lanes_log2);
        if (v > 1e38f) r = make_float2(0x1p-70f, inverse_root(fmaf(z, inv_d, eps * 0x1p-140f)));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = mul2(x[i], make_float2(r.y, r.y));
    return r;
}

// Pairs of a chunk (half layout: of two).
template <typename E, int MODE>
constexpr int pairs_of_chunk() { return MODE == RM_HALF ? Chunk<E>::V : MODE == RM_INTER ? Chunk<E>::V / 2 : 1; }

// One lane's part of a head, normalised if the call asks for it and coded. weight(i) gives the norm's weights of the lane's elements
// 4 i .., other(d) that of element d; `head` is where it was loaded from, unwritten so far; rot(q, c, s) gives cosines and sines
// times m of the pairs of chunk q. Every lane of the warp calls.
template <typename E, int MODE, typename Weight, typename Other, typename Rot>
__device__ __forceinline__ void code_head(const HeadLane<E, MODE>& ln, const HeadArgs& a, const E* head, bool in,
                                          const uint4 (&raw)[2], const Weight& weight, const Other& other, const Rot& rot,
                                          float2 (&x)[Chunk<E>::V]) {
    constexpr int V = Chunk<E>::V, PC = pairs_of_chunk<E, MODE>();
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        float p[V];
        Chunk<E>::unpack(raw[c], p);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) x[c * (V / 2) + i] = make_float2(p[2 * i], p[2 * i + 1]);
    }
    float2 r = make_float2(1.f, 1.f);
    if (a.norm) {
        r = head_norm(x, a.inv_d, a.eps, a.lanes_log2);
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const float4 w = weight(i / 2);
            x[i] = mul2(x[i], make_float2(w.x, w.y));
            x[i + 1] = mul2(x[i + 1], make_float2(w.z, w.w));
        }
    }
    const int half = a.dim / 2;
    if constexpr (MODE == RM_HALF) {
        if (ln.pair) {
            float c[PC], s[PC];
            rot(ln.c[0], c, s);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float2 c2 = make_float2(c[2 * i], c[2 * i + 1]), s2 = make_float2(s[2 * i], s[2 * i + 1]);
                const float2 n2 = make_float2(-s2.x, -s2.y), x1 = x[i], x2 = x[V / 2 + i];
                x[i] = fma2(x1, c2, mul2(x2, n2));
                x[V / 2 + i] = fma2(x2, c2, mul2(x1, s2));
            }
        }
    } else if constexpr (MODE == RM_INTER) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (!ln.live[k] || ln.c[k] * PC >= half) continue;
            float c[PC], s[PC];
            rot(ln.c[k], c, s);
#pragma unroll
            for (int i = 0; i < PC; ++i) {
                float2& z = x[k * PC + i];
                const float2 y = fma2(z, make_float2(c[i], c[i]), mul2(make_float2(z.y, z.x), make_float2(-s[i], s[i])));
                if (ln.c[k] * PC + i < half) z = y;   // (the last chunk may be coded in part)
            }
        }
    } else if constexpr (MODE == RM_SCALAR) {
        // A pair's other element is another lane's: read again, before any lane writes.
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
            const int d = ln.c[i / V] * V + i % V;
            float& y = i & 1 ? x[i / 2].y : x[i / 2].x;
            if (d < a.dim && ln.live[i / V] && in) {
                const int o = d < half ? d + half : d - half;
                float z = to_f(head[o]);
                if (a.norm) z = z * r.x * r.y * other(o);
                float c[1], s[1];
                rot(min(d, o), c, s);
                y = d < half ? y * c[0] - z * s[0] : y * c[0] + z * s[0];
            }
        }
        __syncwarp();
    }
}

// Elements of a lane's chunk c, rounded to E.
template <typename E>
__device__ __forceinline__ uint4 pack_chunk(const float2 (&x)[Chunk<E>::V], int c) {
    constexpr int V = Chunk<E>::V;
    float z[V];
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = i & 1 ? x[c * (V / 2) + i / 2].y : x[c * (V / 2) + i / 2].x;
    return Chunk<E>::pack(z);
}

constexpr int CT_PASSES = 8;     // most heads of a group of lanes in a task
constexpr int CT_THREADS = 256;  // most of a block

// A call's tokens as tasks of single warps: a token, or, of more heads than a warp's groups of lanes take in their passes or in a call
// that is waited for, a part of one.
struct CodeTokens {
    int heads, passes;       // of a token: H queries, K keys, K values; of a group of lanes in a task
    int parts, tasks;        // tasks of a token, of the call
    KvDiv by_parts;
};

// A warp's sines and cosines of its token, and a block's weights.
struct CodeTable {
    float v[2][AP_MAX_PAIRS + 8];
};
struct CodeWeights {
    float4 v[2][4][32];      // of queries and keys: elements 4 i .. of each lane's of a group
};

template <typename E, int MODE>
__device__ __forceinline__ void load_weights(const HeadArgs& a, CodeWeights& w) {
    constexpr int V = Chunk<E>::V;
    if (a.norm)
        for (int e = threadIdx.x; e < 2 * (V / 2) << a.lanes_log2; e += blockDim.x) {
            const int lane = e & ((1 << a.lanes_log2) - 1), i = (e >> a.lanes_log2) % (V / 2), k = (e >> a.lanes_log2) / (V / 2);
            const HeadLane<E, MODE> x(lane, a.D, a.dim);
            const float* f = k ? a.k_weight : a.q_weight;
            const int c = 4 * i / V, d = x.c[c] * V + 4 * i % V;
            w.v[k][i][lane] = f && x.live[c] ? make_float4(f[d], f[d + 1], f[d + 2], f[d + 3]) : make_float4(1.f, 1.f, 1.f, 1.f);
        }
}

// A warp's tasks first, first + step, .. of a call: a table of the token's sines and cosines serves all its heads; the next pass's
// heads are on their way while one is coded. What bounds this on an SM is instructions, not bytes in flight, so that it wants many
// warps that wait for nothing but themselves. (A block to four tokens with a table for all of them, its heads copied ahead through
// shared memory: 4 prompts of 2048 tokens took 24 us, 46 thousand cycles an SM for 21 thousand instructions a scheduler.)
// place(token) is the row that takes it, negative: padding; at(token, row) its place in the cache (element offset). In the table, up
// to four pairs of a chunk lie together, and those of the next chunk, which the next lane reads, behind them.
template <typename E, int MODE, typename Place, typename At>
__device__ __forceinline__ void code_tokens(const HeadArgs& a, const CodeTokens& ct, const CodeWeights& weights, CodeTable& table,
                                            int first, int step, E* ck, E* cv, long long hs, const Place& place, const At& at) {
    constexpr int V = Chunk<E>::V, PC = pairs_of_chunk<E, MODE>(), PV = PC < 4 ? PC : 4;
    const int lane = threadIdx.x & 31, half = a.dim / 2, chunks = (half + PC - 1) / PC;
    const int per = 32 >> a.lanes_log2, u = lane & ((1 << a.lanes_log2) - 1);   // heads of a pass, lane of its head
    const HeadLane<E, MODE> ln(u, a.D, a.dim);
    const int mine = lane >> a.lanes_log2;
    // A task's heads: head hd of its token is at the base of its kind + hd D. (Pointers, which may lie before their buffers.)
    struct Source {
        const E *q, *k, *v;
        int hd0;   // of the warp's first pass
    };
    auto open = [&](int k) {
        uint32_t part;
        const long long tok = ct.by_parts.div((uint32_t)(first + k * step), part);
        Source x;
        x.q = static_cast<const E*>(a.q) + tok * a.q_stride;
        x.k = static_cast<const E*>(a.k) + tok * a.k_stride - a.H * a.D;
        x.v = static_cast<const E*>(a.v) + tok * a.v_stride - (a.H + a.K) * a.D;
        x.hd0 = (int)part * ct.passes * per;
        return x;
    };
    auto source = [&](const Source& x, int hd) { return (hd < a.H ? x.q : hd < a.H + a.K ? x.k : x.v) + hd * a.D; };
    uint4 next[2];
    auto fetch = [&](const Source& x, int p) {
        const int hd = x.hd0 + p * per + mine;
        ln.load(source(x, hd), hd < ct.heads, next);
    };
    for (bool begin = true; first < ct.tasks; first += 32 * step, begin = false) {   // runs of 32 tasks
        const int count = min(32, (ct.tasks - first + step - 1) / step);
        Source src = open(0);
        if (begin) fetch(src, 0);   // beside the rows
        int row = -1, position = 0;   // of the run's task `lane`
        if (lane < count) {
            const int tok = (int)ct.by_parts.div((uint32_t)(first + lane * step));
            row = place(tok);
            position = a.position[tok];
        }
        uint32_t todo = __ballot_sync(0xffffffffu, row >= 0);   // without the padding
        if (todo && !(begin && (todo & 1))) {
            src = open(__ffs(todo) - 1);
            fetch(src, 0);
        }
        while (todo) {
            const int k = __ffs(todo) - 1;
            todo &= todo - 1;
            const int r = __shfl_sync(0xffffffffu, row, k), pos = __shfl_sync(0xffffffffu, position, k);
            const Source x = src;
            if (todo) src = open(__ffs(todo) - 1);
            const long long tok = ct.by_parts.div((uint32_t)(first + k * step));
            if (MODE != RM_NONE) {
                __syncwarp();   // the last task's table has been read
                for (int p = lane; p < half; p += 32) {
                    const float2 c = phase_near(pos, a.turns[p], a.m);
                    const int e = (p % PC / PV * chunks + p / PC) * PV + p % PV;
                    table.v[0][e] = c.x;
                    table.v[1][e] = c.y;
                }
                __syncwarp();
            }
            // Likewise where its heads go.
            E *const dq = static_cast<E*>(a.q_out) + tok * a.H * a.D, *const dk = ck + at(tok, r) - a.H * hs, *const dv = cv + at(tok, r) - (a.H + a.K) * hs;
            const int passes = min(ct.passes, (ct.heads - x.hd0 + per - 1) / per);
#pragma unroll 1
            for (int p = 0; p < passes; ++p) {
                const int hd = x.hd0 + p * per + mine;
                const bool live = hd < ct.heads, value = hd >= a.H + a.K, key = !value && hd >= a.H, coded = live && !value;
                uint4 raw[2] = {next[0], next[1]};
                if (p + 1 < passes) fetch(x, p + 1);
                else if (todo) fetch(src, 0);
                if (__any_sync(0xffffffffu, coded)) {
                    float2 y[V];
                    auto rot = [&](int q, float (&c)[PC], float (&s)[PC]) {
#pragma unroll
                        for (int e = 0; e < PC; e += PV) {
                            const float *fc = &table.v[0][(e / PV * chunks + q) * PV], *fs = &table.v[1][(e / PV * chunks + q) * PV];
                            if constexpr (PV == 4) {
                                const float4 c4 = *reinterpret_cast<const float4*>(fc), s4 = *reinterpret_cast<const float4*>(fs);
                                c[e] = c4.x, c[e + 1] = c4.y, c[e + 2] = c4.z, c[e + 3] = c4.w;
                                s[e] = s4.x, s[e + 1] = s4.y, s[e + 2] = s4.z, s[e + 3] = s4.w;
                            } else if constexpr (PV == 2) {
                                const float2 c2 = *reinterpret_cast<const float2*>(fc), s2 = *reinterpret_cast<const float2*>(fs);
                                c[e] = c2.x, c[e + 1] = c2.y;
                                s[e] = s2.x, s[e + 1] = s2.y;
                            } else {
                                c[e] = *fc;
                                s[e] = *fs;
                            }
                        }
                    };
                    auto weight = [&](int e4) { return weights.v[key][e4][u]; };
                    auto other = [&](int d) {
                        const float* w = key ? a.k_weight : a.q_weight;
                        return w ? w[d] : 1.f;
                    };
                    code_head<E, MODE>(ln, a, MODE == RM_SCALAR && coded ? source(x, hd) : nullptr, coded, raw, weight, other, rot, y);
                    if (coded) {
                        raw[0] = pack_chunk<E>(y, 0);
                        raw[1] = pack_chunk<E>(y, 1);
                    }
                }
                if (!live) continue;
                E* const dst = hd < a.H ? dq + hd * a.D : (value ? dv : dk) + hd * hs;
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (ln.live[c]) *reinterpret_cast<uint4*>(dst + ln.c[c] * V) = raw[c];
            }
        }
    }
}

// Fills in how a call is coded; a.q .. a.norm are the caller's. Returns the rotary mode.
inline int plan_code_tokens(const jpi_kv_handle* h, HeadArgs& a, CodeTokens& ct, int values) {
    const int V = h->bf16 ? 8 : 4;
    int mode = RM_NONE;
    a.D = h->D;
    if (h->rope) {
        a.turns = h->turns;
        a.dim = h->rope_cfg.dim;
        a.m = h->rope_cfg.mscale;
        mode = h->rope_cfg.layout == JPI_ROPE_INTERLEAVED ? RM_INTER : (a.dim / 2) % V == 0 ? RM_HALF : RM_SCALAR;
    }
    a.by_tokens = KvDiv((uint32_t)a.tokens);
    a.lanes_log2 = head_lanes_log2(a.D, V, a.dim, mode);
    a.inv_d = 1.f / (float)a.D;
    ct.heads = std::max(1, a.H + a.K + values);
    const long long n = (long long)a.batch * a.tokens;
    // A token's passes as evenly over tasks as their limit needs, or while there are not two tasks for each of an SM's schedulers.
    const int per = 32 >> a.lanes_log2, all = (ct.heads + per - 1) / per;
    ct.parts = (all + CT_PASSES - 1) / CT_PASSES;
    while (ct.parts < all && n * ct.parts < 8ll * h->num_sms) ++ct.parts;
    ct.passes = (all + ct.parts - 1) / ct.parts;
    ct.parts = (all + ct.passes - 1) / ct.passes;
    ct.by_parts = KvDiv((uint32_t)ct.parts);
    ct.tasks = (int)(n * ct.parts);
    return mode;
}
// Blocks for the tasks: as many tasks for each warp of those that are resident together (`per_sm` blocks).
inline unsigned code_blocks(const jpi_kv_handle* h, const CodeTokens& ct, int threads, int per_sm) {
    const long long warps = threads / 32, all = ((long long)ct.tasks + warps - 1) / warps, most = (long long)h->num_sms * per_sm;
    const long long turns = (all + most - 1) / most;
    return (unsigned)((all + turns - 1) / turns);
}

}  // namespace
}  // namespace jpi
