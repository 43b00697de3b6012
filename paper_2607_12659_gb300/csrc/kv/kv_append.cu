// Rotary coding and cache write (jpi_kv_append).
//
// Pair i of a head, (x1, x2), turns by the angle a = position theta_i:
//   y1 = m (x1 cos a - x2 sin a),  y2 = m (x2 cos a + x1 sin a).
// The table holds theta_i / 2 pi, turns per position, as a fraction of 2^64, so that the phase
// position * turns is an integer product whose wrap-around is the reduction modulo a whole turn:
// exact to 2^-32 turns for any 32-bit position (2^31 * 2^-65 = 2^-34 from the table, 2^-33 from the
// 32 leading bits kept), where a 32-bit angle would be off by a whole turn. sincospif takes it from there.
//
// Bound by memory: every element is read and written once. A block takes tokens in turn; a thread has the same
// units (a 16-byte chunk, or the two chunks of a half-layout pair) of each. The next token's units are on their way
// while this one's sines and cosines are computed, once for all heads, and shared through shared memory; its position
// and row are a token further ahead. (With a block per token, 4 prompts of 2048 tokens of 8 heads of 256 took 21 us, a
// chain of three latencies in each block.)

#include "kv.h"

namespace jpi {
namespace {

enum RopeMode {
    RM_NONE = 0,     // copy
    RM_HALF = 1,     // pairs (d, d + dim / 2), whole chunks of both
    RM_INTER = 2,    // pairs (2 i, 2 i + 1), within a chunk
    RM_SCALAR = 3    // the half layout where dim / 2 is no whole number of chunks: element by element
};

struct AppendArgs {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    const int *position, *row;
    void* q_out;
    void *ck, *cv;
    long long cs, rs, hs;
    int rows;            // of each cache
    int n;               // tokens in all
    KvDiv by_tokens;     // tokens of a request
    int H, K, D;         // H = 0 without queries, K = 0 without keys
    const uint64_t* turns;
    int dim;
    float m;
};

template <typename E>
struct Chunk {   // 16 bytes of E as fp32
    static constexpr int V = 16 / sizeof(E);
    __device__ static __forceinline__ void unpack(uint4 u, float (&x)[V]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 2) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            } else {
                x[i] = __uint_as_float(w[i]);
            }
        }
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[V]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 2) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&b);
            } else {
                w[i] = __float_as_uint(x[i]);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// (cos, sin) of `position` times the pair's turns, times m.
__device__ __forceinline__ float2 phase(int position, uint64_t turns, float m) {
    const uint64_t ph = (uint64_t)(int64_t)position * turns;
    float s, c;
    sincospif((float)(int32_t)(ph >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns in [-1, 1)
    return make_float2(c * m, s * m);
}

constexpr int AP_MAX_PAIRS = 128;   // dim / 2
constexpr int AP_UNITS = 2;         // units of a thread
constexpr int AP_THREADS = 512;     // most of a block

template <typename E, int MODE>
struct AppendUnit {
    int kind = -1;             // 0 query, 1 key, 2 value (copied), -1 none
    int w = 0;                 // chunk, pair of chunks or element of the head
    const E* src = nullptr;    // its head in token 0
    long long dst = 0;         // its head in the destination, without the token
    uint4 r0, r1;
};

template <typename E, int MODE>
__global__ void __launch_bounds__(AP_THREADS) k_kv_append(const __grid_constant__ AppendArgs a) {
    constexpr int V = Chunk<E>::V;
    __shared__ float2 table[2][AP_MAX_PAIRS];
    const int half = a.dim / 2;
    // Units of a coded head: its pairs, then what passes through; of a value head: its chunks.
    const int pairs = MODE == RM_HALF ? half / V : MODE == RM_SCALAR ? half : 0;
    const int per = MODE == RM_HALF ? pairs + (a.D - a.dim) / V : MODE == RM_SCALAR ? a.D - half : a.D / V;
    const int coded = (a.H + a.K) * per, vch = a.D / V, total = coded + (a.v ? a.K * vch : 0);
    int turn = 0;
    for (int u0 = 0; u0 < total; u0 += AP_UNITS * blockDim.x) {
        AppendUnit<E, MODE> un[AP_UNITS];
#pragma unroll
        for (int j = 0; j < AP_UNITS; ++j) {
            const int u = u0 + j * blockDim.x + threadIdx.x;
            if (u < coded) {
                const int h = u / per;
                un[j].kind = h < a.H ? 0 : 1;
                un[j].w = u - h * per;
                un[j].src = h < a.H ? (const E*)a.q + h * a.D : (const E*)a.k + (h - a.H) * a.D;
                un[j].dst = h < a.H ? h * a.D : (h - a.H) * a.hs;
            } else if (u < total) {
                const int h = (u - coded) / vch;
                un[j].kind = 2;
                un[j].w = u - coded - h * vch;
                un[j].src = (const E*)a.v + h * a.D;
                un[j].dst = h * a.hs;
            }
        }
        // The first element of a unit's (first) chunk.
        auto first = [&](const AppendUnit<E, MODE>& x) {
            if (x.kind != 2 && MODE == RM_HALF) return x.w < pairs ? x.w * V : a.dim + (x.w - pairs) * V;
            return x.w * V;
        };
        auto stride = [&](int kind) { return kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride; };
        auto live = [&](int i, int row) { return i < a.n && row >= 0 && row < a.rows; };
        // Token i's units, where it is no padding.
        auto fetch = [&](int i, int row) {
            if (!live(i, row)) return;
#pragma unroll
            for (int j = 0; j < AP_UNITS; ++j) {
                AppendUnit<E, MODE>& x = un[j];
                if (x.kind < 0 || (MODE == RM_SCALAR && x.kind != 2)) continue;
                const E* p = x.src + i * stride(x.kind) + first(x);
                x.r0 = *(const uint4*)p;
                if (MODE == RM_HALF && x.kind != 2 && x.w < pairs) x.r1 = *(const uint4*)(p + half);
            }
        };
        const int step = gridDim.x;
        int i = blockIdx.x;
        int row = i < a.n ? a.row[i] : -1, row1 = i + step < a.n ? a.row[i + step] : -1;
        int pos = i < a.n ? a.position[i] : 0, pos1 = i + step < a.n ? a.position[i + step] : 0;
        fetch(i, row);
        for (; i < a.n; i += step, turn ^= 1) {
            const int row2 = i + 2 * step < a.n ? a.row[i + 2 * step] : -1, pos2 = i + 2 * step < a.n ? a.position[i + 2 * step] : 0;
            float2* cs = table[turn];
            const bool on = live(i, row);   // the same for the whole block
            uint4 c0[AP_UNITS], c1[AP_UNITS];
#pragma unroll
            for (int j = 0; j < AP_UNITS; ++j) {
                c0[j] = un[j].r0;
                c1[j] = un[j].r1;
            }
            fetch(i + step, row1);
            if (MODE != RM_NONE) {
                // (the other table may still be read; this one's readers were through before the last barrier)
                if (on)
                    for (int p = threadIdx.x; p < half; p += blockDim.x) cs[p] = phase(pos, a.turns[p], a.m);
                __syncthreads();
            }
            if (on) {
                const long long b = a.by_tokens.div((uint32_t)i), slot = b * a.cs + row * a.rs;
#pragma unroll
                for (int j = 0; j < AP_UNITS; ++j) {
                    const AppendUnit<E, MODE>& x = un[j];
                    if (x.kind < 0) continue;
                    E* dst = x.kind == 0 ? (E*)a.q_out + (long long)i * a.H * a.D + x.dst
                                         : (x.kind == 1 ? (E*)a.ck : (E*)a.cv) + slot + x.dst;
                    if (x.kind == 2 || MODE == RM_NONE) {
                        *(uint4*)(dst + x.w * V) = c0[j];
                    } else if (MODE == RM_HALF) {
                        const int d = first(x);
                        if (x.w < pairs) {
                            float x1[V], x2[V], y1[V], y2[V];
                            Chunk<E>::unpack(c0[j], x1);
                            Chunk<E>::unpack(c1[j], x2);
#pragma unroll
                            for (int e = 0; e < V; ++e) {
                                const float2 t = cs[d + e];
                                y1[e] = x1[e] * t.x - x2[e] * t.y;
                                y2[e] = x2[e] * t.x + x1[e] * t.y;
                            }
                            *(uint4*)(dst + d) = Chunk<E>::pack(y1);
                            *(uint4*)(dst + d + half) = Chunk<E>::pack(y2);
                        } else {
                            *(uint4*)(dst + d) = c0[j];
                        }
                    } else if (MODE == RM_INTER) {
                        float v[V], y[V];
                        Chunk<E>::unpack(c0[j], v);
#pragma unroll
                        for (int e = 0; e < V; e += 2) {
                            const int p = (x.w * V + e) / 2;
                            const bool in = p < half;
                            const float2 t = in ? cs[p] : make_float2(1.f, 0.f);
                            y[e] = in ? v[e] * t.x - v[e + 1] * t.y : v[e];
                            y[e + 1] = in ? v[e + 1] * t.x + v[e] * t.y : v[e + 1];
                        }
                        *(uint4*)(dst + x.w * V) = Chunk<E>::pack(y);
                    } else {
                        const E* src = x.src + i * stride(x.kind);
                        if (x.w < half) {
                            const float x1 = to_f(src[x.w]), x2 = to_f(src[x.w + half]);
                            const float2 t = cs[x.w];
                            put(dst + x.w, x1 * t.x - x2 * t.y);
                            put(dst + x.w + half, x2 * t.x + x1 * t.y);
                        } else {
                            dst[x.w + half] = src[x.w + half];
                        }
                    }
                }
            }
            row = row1;
            pos = pos1;
            row1 = row2;
            pos1 = pos2;
        }
        if (MODE != RM_NONE) __syncthreads();   // the next units' tokens begin with a table that may still be read
    }
}

template <typename E>
jpi_status launch(const AppendArgs& a, int mode, int num_sms, cudaStream_t st) {
    constexpr int V = Chunk<E>::V;
    const int half = a.dim / 2;
    const int per = mode == RM_HALF ? half / V + (a.D - a.dim) / V : mode == RM_SCALAR ? a.D - half : a.D / V;
    const int total = (a.H + a.K) * per + (a.v ? a.K * (a.D / V) : 0);
    int threads = (total + AP_UNITS - 1) / AP_UNITS;
    threads = threads > AP_THREADS ? AP_THREADS : (threads + 31) / 32 * 32;
    const long long most = (long long)num_sms * (1024 / threads);
    const long long grid = a.n < most ? a.n : most;
    return kv_start(mode == RM_NONE ? k_kv_append<E, RM_NONE>
                                    : mode == RM_HALF ? k_kv_append<E, RM_HALF>
                                                      : mode == RM_INTER ? k_kv_append<E, RM_INTER> : k_kv_append<E, RM_SCALAR>,
                    grid, threads, 0, false, st, a);
}

}  // namespace

jpi_status launch_kv_append(const jpi_kv_handle* h, const void* q, long long q_stride, const void* k, long long k_stride,
                            const void* v, long long v_stride, const int* position, const int* row, int batch,
                            int tokens, void* q_out, const jpi_kv_cache* cache, cudaStream_t st) {
    AppendArgs a = {};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.position = position;
    a.row = row;
    a.q_out = q_out;
    a.rows = 0x7fffffff;
    if (cache) {
        a.ck = cache->k;
        a.cv = cache->v;
        a.cs = cache->cache_stride;
        a.rs = cache->row_stride;
        a.hs = cache->head_stride;
        a.rows = cache->rows;
    }
    a.n = batch * tokens;   // (the maxima keep it below 2^28)
    a.by_tokens = KvDiv((uint32_t)tokens);
    a.H = q ? h->H : 0;
    a.K = k ? h->K : 0;
    a.D = h->D;
    int mode = RM_NONE;
    if (h->rope) {
        a.turns = h->turns;
        a.dim = h->rope_cfg.dim;
        a.m = h->rope_cfg.mscale;
        const int V = h->bf16 ? 8 : 4;
        mode = h->rope_cfg.layout == JPI_ROPE_INTERLEAVED ? RM_INTER : (a.dim / 2) % V == 0 ? RM_HALF : RM_SCALAR;
    }
    return h->bf16 ? launch<__nv_bfloat16>(a, mode, h->num_sms, st) : launch<float>(a, mode, h->num_sms, st);
}

}  // namespace jpi
