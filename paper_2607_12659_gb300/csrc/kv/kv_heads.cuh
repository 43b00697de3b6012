// Heads held by groups of lanes: the norm of a head and its rotary coding in registers (kv_append_normed.cu, kv8_append.cu).
//
// A head of D elements is C = D / V chunks of 16 bytes. A group of G lanes (a power of two, at most a warp) holds it, two
// chunks a lane: in the half layout a pair's two chunks, so that a lane has both elements of each of its pairs and the
// rotation needs no exchange; else two neighbours. The sum of squares is a sum over the group by shuffles.
#pragma once

#include "kv_code.cuh"

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

// One lane's part of a head, normalised (with `weight`, in memory that every lane can read, or NULL) and coded. `head` is
// where it was loaded from, unwritten so far; rot(pair) gives (cos, sin) times m. Every lane of the warp calls.
template <typename E, int MODE, typename Rot>
__device__ __forceinline__ void code_head(const HeadLane<E, MODE>& ln, const HeadArgs& a, const E* head, bool in,
                                          const uint4 (&raw)[2], bool norm, const float* weight, const Rot& rot,
                                          float (&y)[2 * Chunk<E>::V]) {
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
        for (int i = 0; i < 2 * V; ++i) {
            x[i] = x[i] * r.x * r.y;
            if (weight && ln.live[i / V]) x[i] *= weight[ln.c[i / V] * V + i % V];
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
                if (norm) {
                    z = z * r.x * r.y;
                    if (weight) z *= weight[o];
                }
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

constexpr int CT_TOKENS = 8;    // most tokens of a block
constexpr int CT_PASSES = 4;    // heads of a group of lanes that are on their way together
constexpr int CT_THREADS = 256;

struct CodeTokens {
    int tt;               // tokens of a block
    KvDiv by_heads;       // rows of a token: H queries, K keys, K values
    int heads;
};

struct CodeSmem {
    float2 table[CT_TOKENS][AP_MAX_PAIRS + 8];
    float weight[2][256];
    int2 token[CT_TOKENS];   // (row, position)
};

// The tokens tt * block, .. of a call: rotary tables of all of them, then their heads in turn. place(token) is the row that
// takes it, negative: padding; at(token, row) its place in the cache (element offset). A table is laid out so that the
// lanes of a group, which read the same pair of consecutive chunks, read side by side.
template <typename E, int MODE, typename Place, typename At>
__device__ __forceinline__ void code_tokens(const HeadArgs& a, const CodeTokens& ct, CodeSmem& sm, int block, E* ck, E* cv,
                                            long long hs, const Place& place, const At& at) {
    constexpr int V = Chunk<E>::V, PC = MODE == RM_HALF ? V : MODE == RM_INTER ? V / 2 : 1;
    const int t = threadIdx.x, nth = blockDim.x, half = a.dim / 2, chunks = (half + PC - 1) / PC;
    const int tok0 = block * ct.tt, nt = min(ct.tt, a.batch * a.tokens - tok0), rows = nt * ct.heads;
    const int groups = nth >> a.lanes_log2, grp = t >> a.lanes_log2;
    const HeadLane<E, MODE> ln(t & ((1 << a.lanes_log2) - 1), a.D, a.dim);
    auto entry = [&](int p) { return p % PC * chunks + p / PC; };
    for (int r0 = 0; r0 < rows; r0 += CT_PASSES * groups) {
        uint4 raw[CT_PASSES][2];
        const E* src[CT_PASSES];
#pragma unroll
        for (int p = 0; p < CT_PASSES; ++p) {
            const int r = r0 + p * groups + grp;
            uint32_t h;
            const long long tok = tok0 + ct.by_heads.div((uint32_t)r, h);
            const int hd = (int)h;
            src[p] = hd < a.H ? static_cast<const E*>(a.q) + tok * a.q_stride + hd * a.D
                              : hd < a.H + a.K ? static_cast<const E*>(a.k) + tok * a.k_stride + (hd - a.H) * a.D
                                               : static_cast<const E*>(a.v) + tok * a.v_stride + (hd - a.H - a.K) * a.D;
            ln.load(src[p], r < rows, raw[p]);
        }
        if (r0 == 0) {   // beside the first loads
            if (t < nt) sm.token[t] = make_int2(place(tok0 + t), a.position[tok0 + t]);
            if (a.norm)
                for (int d = t; d < a.D; d += nth) {
                    sm.weight[0][d] = a.q_weight ? a.q_weight[d] : 1.f;
                    sm.weight[1][d] = a.k_weight ? a.k_weight[d] : 1.f;
                }
            if (MODE != RM_NONE)
                for (int e = t; e < nt * half; e += nth) {
                    const int i = e / half, p = e - i * half;
                    sm.table[i][entry(p)] = phase_near(a.position[tok0 + i], a.turns[p], a.m);
                }
            __syncthreads();
        }
#pragma unroll
        for (int p = 0; p < CT_PASSES; ++p) {
            if (r0 + p * groups >= rows) break;   // (the same for the block)
            const int r = r0 + p * groups + grp;
            const bool in = r < rows;
            uint32_t h;
            const int i = in ? (int)ct.by_heads.div((uint32_t)r, h) : 0, hd = in ? (int)h : 0;
            const bool value = hd >= a.H + a.K, key = !value && hd >= a.H;
            float y[2 * V];
            auto rot = [&](int pr) { return sm.table[i][entry(pr)]; };
            code_head<E, MODE>(ln, a, src[p], in && !value, raw[p], a.norm, sm.weight[key], rot, y);
            const int row = sm.token[i].x;
            if (!in || row < 0) continue;
            const long long tok = tok0 + i;
            E* dst = hd < a.H ? static_cast<E*>(a.q_out) + (tok * a.H + hd) * a.D
                              : (value ? cv + (hd - a.H - a.K) * hs : ck + (hd - a.H) * hs) + at(tok, row);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (!ln.live[c]) continue;
                float z[V];
#pragma unroll
                for (int e = 0; e < V; ++e) z[e] = y[c * V + e];
                *reinterpret_cast<uint4*>(dst + ln.c[c] * V) = value ? raw[p][c] : Chunk<E>::pack(z);
            }
        }
    }
}

// Fills in how a call is coded; a.q .. a.norm are the caller's.
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
    ct.heads = a.H + a.K + values;
    ct.by_heads = KvDiv((uint32_t)(ct.heads > 0 ? ct.heads : 1));
    const long long n = (long long)a.batch * a.tokens;
    // As many tokens as a block's loads in flight hold, while there are two blocks an SM.
    const int groups = CT_THREADS >> a.lanes_log2;
    ct.tt = 1;
    while (ct.tt < CT_TOKENS && 2 * ct.tt * ct.heads <= CT_PASSES * groups && n >= 4ll * ct.tt * h->num_sms) ct.tt *= 2;
    const int want = ((ct.tt * ct.heads) << a.lanes_log2) + 31;
    *threads = want >= CT_THREADS ? CT_THREADS : want < 64 ? 64 : want / 32 * 32;
    return mode;
}

}  // namespace
}  // namespace jpi
