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

__device__ __forceinline__ float group_sum(float x, int lanes_log2) {
    for (int i = 0; i < lanes_log2; ++i) x += __shfl_xor_sync(0xffffffffu, x, 1 << i);
    return x;
}

// The factors (first, second) that make a head's elements x (those of one lane) x / sqrt(mean(x^2) + eps). Of heads whose squares
// pass fp32's range the first is 2^-70, else it is 1. Every lane of the warp calls.
template <int N>
__device__ __forceinline__ float2 head_norm(const float (&x)[N], int D, float eps, int lanes_log2) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(x[i], x[i], s);
    s = group_sum(s, lanes_log2);
    float2 r = make_float2(1.f, 1.f / sqrtf(s / (float)D + eps));
    if (__any_sync(0xffffffffu, s > 1e38f)) {
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) z = fmaf(x[i] * 0x1p-70f, x[i] * 0x1p-70f, z);
        z = group_sum(z, lanes_log2);
        if (s > 1e38f) r = make_float2(0x1p-70f, 1.f / sqrtf(z / (float)D));   // (eps is less than a rounding here)
    }
    return r;
}

// One lane's part of a head, normalised if the call asks for it and coded. weight(i) gives the norm's weights of the lane's elements
// 4 i .., other(d) that of element d; `head` is where it was loaded from, unwritten so far; rot(pair) gives (cos, sin)
// times m. Every lane of the warp calls.
template <typename E, int MODE, typename Weight, typename Other, typename Rot>
__device__ __forceinline__ void code_head(const HeadLane<E, MODE>& ln, const HeadArgs& a, const E* head, bool in,
                                          const uint4 (&raw)[2], const Weight& weight, const Other& other, const Rot& rot,
                                          float (&y)[2 * Chunk<E>::V]) {
    const bool norm = a.norm;
    constexpr int V = Chunk<E>::V;
    float x[2 * V];
    {
        float p[2][V];
        Chunk<E>::unpack(raw[0], p[0]);
        Chunk<E>::unpack(raw[1], p[1]);
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) x[i] = p[i / V][i % V];
    }
    float2 r = make_float2(1.f, 1.f);
    if (norm) {
        r = head_norm(x, a.D, a.eps, a.lanes_log2);
#pragma unroll
        for (int i = 0; i < 2 * V; i += 4) {
            const float4 w = weight(i / 4);
            x[i] = x[i] * r.x * r.y * w.x;
            x[i + 1] = x[i + 1] * r.x * r.y * w.y;
            x[i + 2] = x[i + 2] * r.x * r.y * w.z;
            x[i + 3] = x[i + 3] * r.x * r.y * w.w;
        }
    }
    const int half = a.dim / 2;
    if (MODE == RM_HALF && ln.pair) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float2 c = rot(ln.c[0] * V + i);
            y[i] = x[i] * c.x - x[V + i] * c.y;
            y[V + i] = x[V + i] * c.x + x[i] * c.y;
        }
    } else if (MODE == RM_INTER) {
#pragma unroll
        for (int i = 0; i < 2 * V; i += 2) {
            const int p = (ln.c[i / V] * V + i % V) / 2;
            const bool turn = p < half && ln.live[i / V];
            const float2 c = turn ? rot(p) : make_float2(1.f, 0.f);
            y[i] = turn ? x[i] * c.x - x[i + 1] * c.y : x[i];
            y[i + 1] = turn ? x[i + 1] * c.x + x[i] * c.y : x[i + 1];
        }
    } else if (MODE == RM_SCALAR) {
        // A pair's other element is another lane's: read again, before any lane writes.
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
            const int d = ln.c[i / V] * V + i % V;
            const bool turn = d < a.dim && ln.live[i / V] && in;
            y[i] = x[i];
            if (turn) {
                const int o = d < half ? d + half : d - half;
                float z = to_f(head[o]);
                if (norm) z = z * r.x * r.y * other(o);
                const float2 c = rot(d < half ? d : o);
                y[i] = d < half ? x[i] * c.x - z * c.y : x[i] * c.x + z * c.y;
            }
        }
        __syncwarp();
    } else {
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) y[i] = x[i];
    }
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
    float2 table[2][CT_TOKENS][AP_MAX_PAIRS + 8];
    float4 weight[2][4][32];          // of queries and keys: elements 4 i .. of each lane's of a group
    int2 token[CT_RUN][CT_TOKENS];    // (row, position)
};

// Takes tasks first, first + step, .. of a call. Their heads are copied asynchronously into shared memory, each thread's chunks
// into places of its own, two tasks ahead of the one whose sines, cosines and norms are computed; a table of those of a task's tokens
// serves all its heads. place(token) is the row that takes it, negative: padding; at(token, row) its place in the cache (element
// offset). A table is laid out so that the lanes of a group, which read the same pair of consecutive chunks, read side by side.
template <typename E, int MODE, typename Place, typename At>
__device__ __forceinline__ void code_tokens(const HeadArgs& a, const CodeTokens& ct, CodeSmem& sm, uint4* stage, int first, int step,
                                            E* ck, E* cv, long long hs, const Place& place, const At& at) {
    constexpr int V = Chunk<E>::V, PC = MODE == RM_HALF ? V : MODE == RM_INTER ? V / 2 : 1;
    const int t = threadIdx.x, nth = blockDim.x, half = a.dim / 2, chunks = (half + PC - 1) / PC;
    const int groups = nth >> a.lanes_log2, grp = t >> a.lanes_log2, u = t & ((1 << a.lanes_log2) - 1), n = a.batch * a.tokens;
    const HeadLane<E, MODE> ln(u, a.D, a.dim);
    auto entry = [&](int p) { return p % PC * chunks + p / PC; };
    auto slot = [&](int k, int p, int c) { return ((k % CT_STAGES * ct.passes + p) * 2 + c) * nth + t; };
    struct Task {
        int tok0, nt, r0, rows;   // tokens; rows r0 .. rows - 1 of (token, head)
    };
    auto task_of = [&](int k) {   // the run's k-th
        uint32_t part;
        Task x;
        x.tok0 = (int)ct.by_parts.div((uint32_t)(first + k * step), part) * ct.tt;
        x.nt = min(ct.tt, n - x.tok0);
        x.r0 = (int)part * ct.passes * groups;
        x.rows = min(x.nt * ct.heads, x.r0 + ct.passes * groups);
        return x;
    };
    // A row's token of the task and head.
    auto head_of = [&](int r, int& i) {
        uint32_t h;
        i = (int)ct.by_heads.div((uint32_t)r, h);
        return (int)h;
    };
    auto source = [&](long long tok, int hd) {
        return hd < a.H ? static_cast<const E*>(a.q) + tok * a.q_stride + hd * a.D
                        : hd < a.H + a.K ? static_cast<const E*>(a.k) + tok * a.k_stride + (hd - a.H) * a.D
                                         : static_cast<const E*>(a.v) + tok * a.v_stride + (hd - a.H - a.K) * a.D;
    };
    auto fetch = [&](int k, int count, bool known) {
        if (k < count) {
            const Task x = task_of(k);
            for (int p = 0; p < ct.passes; ++p) {
                const int r = x.r0 + p * groups + grp;
                if (r >= x.rows) break;
                int i;
                const int hd = head_of(r, i);
                if (known && sm.token[k][i].x < 0) continue;
                const E* src = source(x.tok0 + i, hd);
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (ln.live[c]) ptx::cp_async_16(ptx::smem_u32(stage + slot(k, p, c)), src + ln.c[c] * V, true);
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
            const int k = e / ct.tt, i = e - k * ct.tt;
            const Task x = task_of(k);
            if (i < x.nt) sm.token[k][i] = make_int2(place(x.tok0 + i), a.position[x.tok0 + i]);
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
            const Task x = task_of(k);
            turn ^= 1;   // the other table may still be read; this one's readers are past the last barrier
            if (MODE != RM_NONE) {
                for (int e = t; e < x.nt * half; e += nth) {
                    const int i = e / half, p = e - i * half;
                    if (sm.token[k][i].x >= 0) sm.table[turn][i][entry(p)] = phase_near(sm.token[k][i].y, a.turns[p], a.m);
                }
                __syncthreads();
            }
            asm volatile("cp.async.wait_group 2;" ::: "memory");
            for (int p = 0; p < ct.passes; ++p) {
                if (x.r0 + p * groups >= x.rows) break;   // (the same for the block)
                const int r = x.r0 + p * groups + grp;
                int i;
                int hd = head_of(min(r, x.rows - 1), i);
                const bool live = r < x.rows && sm.token[k][i].x >= 0;
                if (!__any_sync(0xffffffffu, live)) continue;
                const bool value = hd >= a.H + a.K, key = !value && hd >= a.H;
                uint4 raw[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) raw[c] = live && ln.live[c] ? stage[slot(k, p, c)] : make_uint4(0, 0, 0, 0);
                float y[2 * V];
                auto rot = [&](int pr) { return sm.table[turn][i][entry(pr)]; };
                auto weight = [&](int e4) { return sm.weight[key][e4][u]; };
                auto other = [&](int d) { return (key ? a.k_weight : a.q_weight) ? (key ? a.k_weight : a.q_weight)[d] : 1.f; };
                const E* src = source(x.tok0 + i, hd);
                code_head<E, MODE>(ln, a, src, live && !value, raw, weight, other, rot, y);
                if (!live) continue;
                const int row = sm.token[k][i].x;
                const long long tok = x.tok0 + i;
                E* dst = hd < a.H ? static_cast<E*>(a.q_out) + (tok * a.H + hd) * a.D
                                  : (value ? cv + (hd - a.H - a.K) * hs : ck + (hd - a.H) * hs) + at(tok, row);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (!ln.live[c]) continue;
                    float z[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) z[e] = y[c * V + e];
                    *reinterpret_cast<uint4*>(dst + ln.c[c] * V) = value ? raw[c] : Chunk<E>::pack(z);
                }
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
