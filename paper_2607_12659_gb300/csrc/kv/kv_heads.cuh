// Heads held by groups of lanes: the norm of a head and its rotary coding in registers (kv_append_normed.cu, kv8_append.cu).
//
// A head of D elements is C = D / V chunks of 16 bytes. A group of G lanes (a power of two, at most a warp) holds it, two
// chunks a lane: in the half layout a pair's two chunks, so that a lane has both elements of each of its pairs and the
// rotation needs no exchange; else two neighbours. The sum of squares is a sum over the group by shuffles.
#pragma once

#include "kv_code.cuh"
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
    float eps;
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

// Two fp32 numbers by one instruction.
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

__device__ __forceinline__ float group_sum(float x, int lanes_log2) {
    for (int i = 0; i < lanes_log2; ++i) x += __shfl_xor_sync(0xffffffffu, x, 1 << i);
    return x;
}

// Makes a head's elements x (those of one lane) x / sqrt(mean(x^2) + eps); returns the factors that did it, one after the other. Of heads
// whose squares pass fp32's range the first is 2^-70, else it is 1. Every lane of the warp calls.
template <int N>
__device__ __forceinline__ float2 head_norm(float2 (&x)[N], int D, float eps, int lanes_log2) {
    float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i) s2 = fma2(x[i], x[i], s2);
    const float s = group_sum(s2.x + s2.y, lanes_log2);
    float2 r = make_float2(1.f, 1.f / sqrtf(s / (float)D + eps));
    if (__any_sync(0xffffffffu, s > 1e38f)) {
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 y = make_float2(x[i].x * 0x1p-70f, x[i].y * 0x1p-70f);
            z = fmaf(y.x, y.x, fmaf(y.y, y.y, z));
            if (s > 1e38f) x[i] = y;
        }
        z = group_sum(z, lanes_log2);
        if (s > 1e38f) r = make_float2(0x1p-70f, 1.f / sqrtf(z / (float)D));   // (eps is less than a rounding here)
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
        r = head_norm(x, a.D, a.eps, a.lanes_log2);
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

constexpr int CT_TOKENS = 4;    // most tokens of a task
constexpr int CT_PASSES = 4;    // most heads of a group of lanes in a task
constexpr int CT_STAGES = 3;    // tasks in hand
constexpr int CT_RUN = 16;      // tasks whose rows and positions are read together
constexpr int CT_THREADS = 256;

// A call's tokens as tasks: `tt` tokens, or, of more heads than the groups of lanes hold in their passes, a part of one token's.
struct CodeTokens {
    int tt, heads, passes;   // heads of a token: H queries, K keys, K values
    int parts, tasks;        // tasks of a token, of the call
    KvDiv by_heads, by_parts;
};

struct CodeSmem {
    float table[2][CT_TOKENS][2][AP_MAX_PAIRS + 8];   // cosines and sines of the tokens of this task and the last
    float4 weight[2][4][32];          // of queries and keys: elements 4 i .. of each lane's of a group
    int2 token[CT_RUN][CT_TOKENS];    // (row, position)
};

// Takes tasks first, first + step, .. of a call. Their heads are copied asynchronously into shared memory, each thread's chunks
// into places of its own, two tasks ahead of the one whose sines, cosines and norms are computed; a table of those of a task's tokens
// serves all its heads. place(token) is the row that takes it, negative: padding; at(token, row) its place in the cache (element
// offset). In a table, up to four pairs of a chunk lie together, and those of the next chunk, which the next lane reads, behind them.
template <typename E, int MODE, typename Place, typename At>
__device__ __forceinline__ void code_tokens(const HeadArgs& a, const CodeTokens& ct, CodeSmem& sm, uint4* stage, int first, int step,
                                            E* ck, E* cv, long long hs, const Place& place, const At& at) {
    constexpr int V = Chunk<E>::V, PC = pairs_of_chunk<E, MODE>(), PV = PC < 4 ? PC : 4;
    const int t = threadIdx.x, nth = blockDim.x, half = a.dim / 2, chunks = (half + PC - 1) / PC;
    const int groups = nth >> a.lanes_log2, grp = t >> a.lanes_log2, u = t & ((1 << a.lanes_log2) - 1), n = a.batch * a.tokens;
    const HeadLane<E, MODE> ln(u, a.D, a.dim);
    auto entry = [&](int p) { return (p % PC / PV * chunks + p / PC) * PV + p % PV; };
    const uint32_t mine = ptx::smem_u32(stage) + 16 * t;
    auto slot = [&](int k, int p, int c) { return ((k % CT_STAGES * ct.passes + p) * 2 + c) * nth; };
    // The group's heads of a task, pass by pass: the same of every task where a task has whole tokens.
    struct Unit {
        int kind;          // 0 query, 1 key, 2 value, -1 none
        int i;             // token of the task
        const E* src;      // of a task that begins with token 0
        long long stride;
        E* dst;            // without the token of a query, or the row of a key or value
    } un[CT_PASSES];
    auto set_units = [&](int part) {
#pragma unroll
        for (int p = 0; p < CT_PASSES; ++p) {
            const int r = (part * ct.passes + p) * groups + grp;
            uint32_t h;
            Unit& x = un[p];
            x.i = (int)ct.by_heads.div((uint32_t)r, h);
            int hd = (int)h;
            x.kind = p >= ct.passes || x.i >= ct.tt ? -1 : hd < a.H ? 0 : hd < a.H + a.K ? 1 : 2;
            hd -= x.kind == 1 ? a.H : x.kind == 2 ? a.H + a.K : 0;
            x.stride = x.kind == 1 ? a.k_stride : x.kind == 2 ? a.v_stride : a.q_stride;
            x.src = static_cast<const E*>(x.kind == 1 ? a.k : x.kind == 2 ? a.v : a.q) + x.i * x.stride + hd * a.D;
            x.dst = x.kind == 0 ? static_cast<E*>(a.q_out) + ((long long)x.i * a.H + hd) * a.D : (x.kind == 1 ? ck : cv) + hd * hs;
        }
    };
    set_units(0);
    // Of the run's k-th task: its first token and tokens, and its units.
    auto open = [&](int k, int& tok0) {
        uint32_t part;
        tok0 = (int)ct.by_parts.div((uint32_t)(first + k * step), part) * ct.tt;
        if (ct.parts > 1) set_units((int)part);
        return min(ct.tt, n - tok0);
    };
    auto fetch = [&](int k, int count, bool known) {
        if (k < count) {
            int tok0;
            const int nt = open(k, tok0);
#pragma unroll
            for (int p = 0; p < CT_PASSES; ++p) {
                const Unit& x = un[p];
                if (x.kind < 0 || x.i >= nt || (known && sm.token[k][x.i].x < 0)) continue;
                const E* src = x.src + tok0 * x.stride;
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (ln.live[c]) ptx::cp_async_16(mine + 16 * slot(k, p, c), src + ln.c[c] * V, true);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int turn = 0;
    for (bool begin = true; first < ct.tasks; first += CT_RUN * step, begin = false) {
        const int count = min(CT_RUN, (ct.tasks - first + step - 1) / step);
        if (begin) fetch(0, count, false);   // the first task's heads on their way beside its rows
        __syncthreads();                     // the last run's tokens have been read
        for (int e = t; e < count * ct.tt; e += nth) {
            const int k = e / ct.tt, tok = (int)ct.by_parts.div((uint32_t)(first + k * step)) * ct.tt + e - k * ct.tt;
            if (tok < n) sm.token[k][e - k * ct.tt] = make_int2(place(tok), a.position[tok]);
        }
        if (begin && a.norm)
            for (int e = t; e < 2 * (V / 2) << a.lanes_log2; e += nth) {
                const int lane = e & ((1 << a.lanes_log2) - 1), i = (e >> a.lanes_log2) % (V / 2), k = (e >> a.lanes_log2) / (V / 2);
                const HeadLane<E, MODE> x(lane, a.D, a.dim);
                const float* w = k ? a.k_weight : a.q_weight;
                const int c = 4 * i / V, d = x.c[c] * V + 4 * i % V;
                sm.weight[k][i][lane] = w && x.live[c] ? make_float4(w[d], w[d + 1], w[d + 2], w[d + 3]) : make_float4(1.f, 1.f, 1.f, 1.f);
            }
        __syncthreads();
        if (!begin) fetch(0, count, true);
        fetch(1, count, true);
        for (int k = 0; k < count; ++k) {
            fetch(k + 2, count, true);
            int tok0;
            const int nt = open(k, tok0);
            turn ^= 1;   // the other table may still be read; this one's readers are past the last barrier
            if (MODE != RM_NONE) {
                for (int e = t; e < nt * half; e += nth) {
                    const int i = e / half, p = e - i * half;
                    if (sm.token[k][i].x < 0) continue;
                    const float2 c = phase_near(sm.token[k][i].y, a.turns[p], a.m);
                    sm.table[turn][i][0][entry(p)] = c.x;
                    sm.table[turn][i][1][entry(p)] = c.y;
                }
                __syncthreads();
            }
            asm volatile("cp.async.wait_group 2;" ::: "memory");
#pragma unroll
            for (int p = 0; p < CT_PASSES; ++p) {
                if (p >= ct.passes) break;
                const Unit& x = un[p];
                const int2 token = x.kind >= 0 && x.i < nt ? sm.token[k][x.i] : make_int2(-1, 0);
                const bool live = token.x >= 0, coded = live && x.kind != 2;
                uint4 raw[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) raw[c] = live && ln.live[c] ? stage[slot(k, p, c) + t] : make_uint4(0, 0, 0, 0);
                if (__any_sync(0xffffffffu, coded)) {
                    const int i = live ? x.i : 0;
                    float2 y[V];
                    auto rot = [&](int q, float (&c)[PC], float (&s)[PC]) {
#pragma unroll
                        for (int e = 0; e < PC; e += PV) {
                            const float *fc = &sm.table[turn][i][0][(e / PV * chunks + q) * PV], *fs = &sm.table[turn][i][1][(e / PV * chunks + q) * PV];
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
                    auto weight = [&](int e4) { return sm.weight[x.kind == 1][e4][u]; };
                    auto other = [&](int d) {
                        const float* w = x.kind == 1 ? a.k_weight : a.q_weight;
                        return w ? w[d] : 1.f;
                    };
                    code_head<E, MODE>(ln, a, x.src + tok0 * x.stride, coded, raw, weight, other, rot, y);
                    if (coded) {
                        raw[0] = pack_chunk<E>(y, 0);
                        raw[1] = pack_chunk<E>(y, 1);
                    }
                }
                if (!live) continue;
                E* dst = x.dst + (x.kind == 0 ? (long long)tok0 * a.H * a.D : at(tok0 + x.i, token.x));
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (ln.live[c]) *reinterpret_cast<uint4*>(dst + ln.c[c] * V) = raw[c];
            }
        }
        ptx::cp_async_wait_all();   // (empty groups)
    }
}

// Fills in how a call is coded; a.q .. a.norm are the caller's. Returns the rotary mode.
inline int plan_code_tokens(const jpi_kv_handle* h, HeadArgs& a, CodeTokens& ct, int values, int* threads) {
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
    ct.heads = std::max(1, a.H + a.K + values);
    ct.by_heads = KvDiv((uint32_t)ct.heads);
    const long long n = (long long)a.batch * a.tokens;
    // Tokens of a task: as many as its passes hold, while there are two tasks an SM.
    const int groups = CT_THREADS >> a.lanes_log2;
    ct.tt = 1;
    while (ct.tt < CT_TOKENS && 2 * ct.tt * ct.heads <= CT_PASSES * groups && n >= 4ll * ct.tt * h->num_sms) ct.tt *= 2;
    ct.passes = std::min(CT_PASSES, (ct.tt * ct.heads + groups - 1) / groups);
    ct.parts = (ct.tt * ct.heads + ct.passes * groups - 1) / (ct.passes * groups);
    ct.by_parts = KvDiv((uint32_t)ct.parts);
    ct.tasks = (int)((n + ct.tt - 1) / ct.tt * ct.parts);
    *threads = ct.parts > 1 || ct.passes > 1 ? CT_THREADS : std::max(64, ((ct.tt * ct.heads << a.lanes_log2) + 31) / 32 * 32);
    return mode;
}
inline size_t code_smem(const CodeTokens& ct, int threads) { return (size_t)CT_STAGES * ct.passes * 2 * threads * 16; }
// Blocks that are resident together, by shared memory (to 190 KB of an SM) and threads.
inline long long code_blocks(const jpi_kv_handle* h, size_t smem, int threads) {
    return (long long)h->num_sms * std::max<long long>(1, std::min<long long>(1536 / threads, (190 << 10) / (long long)(smem + sizeof(CodeSmem) + 2048)));
}

}  // namespace
}  // namespace jpi
