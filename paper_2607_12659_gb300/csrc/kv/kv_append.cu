// Rotary coding and cache write (jpi_kv_append).
//
// Pair i of a head, (x1, x2), turns by the angle a = position theta_i:
//   y1 = m (x1 cos a - x2 sin a),  y2 = m (x2 cos a + x1 sin a).
// The table holds theta_i / 2 pi, turns per position, as a fraction of 2^64, so that the phase
// position * turns is an integer product whose wrap-around is the reduction modulo a whole turn:
// exact to 2^-32 turns for any 32-bit position (2^31 * 2^-65 = 2^-34 from the table, 2^-33 from the
// 32 leading bits kept), where a 32-bit angle would be off by a whole turn. sincospif takes it from there.
//
// Bound by memory: every element is read and written once. One block per token: its units (a
// 16-byte chunk, or the two chunks of a half-layout pair) are loaded first, the token's sines and cosines
// computed while they are in flight, once for all heads, and shared through shared memory.

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
    int tokens;          // per request
    long long n;         // tokens in all
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
constexpr int AP_UNITS = 4;         // units of a thread in flight

template <typename E, int MODE>
__global__ void k_kv_append(const __grid_constant__ AppendArgs a) {
    constexpr int V = Chunk<E>::V;
    __shared__ float2 cs[AP_MAX_PAIRS];
    const int half = a.dim / 2;
    // Units of a coded head: its pairs, then what passes through; of a value head: its chunks.
    const int pairs = MODE == RM_HALF ? half / V : MODE == RM_SCALAR ? half : 0;
    const int per = MODE == RM_HALF ? pairs + (a.D - a.dim) / V : MODE == RM_SCALAR ? a.D - half : a.D / V;
    const int coded = (a.H + a.K) * per, vch = a.D / V;
    const int total = coded + (a.v ? a.K * vch : 0);
    for (long long i = blockIdx.x; i < a.n; i += gridDim.x) {
        const int row = a.row[i];
        if (row < 0 || row >= a.rows) continue;   // padding (the same for the whole block)
        const int position = a.position[i];
        const long long b = i / a.tokens;
        E* krow = (E*)a.ck + b * a.cs + row * a.rs;
        E* vrow = (E*)a.cv + b * a.cs + row * a.rs;
        bool table = false;
        for (int u0 = threadIdx.x; u0 - (int)threadIdx.x < total; u0 += AP_UNITS * blockDim.x) {
            uint4 r0[AP_UNITS], r1[AP_UNITS];
            const E* src[AP_UNITS];
            E* dst[AP_UNITS];
            int w[AP_UNITS];   // unit within its head; -1 for a value chunk, -2 past the end
#pragma unroll
            for (int j = 0; j < AP_UNITS; ++j) {
                const int u = u0 + j * blockDim.x;
                w[j] = -2;
                src[j] = nullptr;
                dst[j] = nullptr;
                r0[j] = r1[j] = make_uint4(0, 0, 0, 0);
                if (u < coded) {
                    const int h = u / per;
                    w[j] = u - h * per;
                    src[j] = h < a.H ? (const E*)a.q + i * a.q_stride + h * a.D : (const E*)a.k + i * a.k_stride + (h - a.H) * a.D;
                    dst[j] = h < a.H ? (E*)a.q_out + (i * a.H + h) * a.D : krow + (h - a.H) * a.hs;
                    if (MODE == RM_HALF) {
                        const int d = w[j] < pairs ? w[j] * V : a.dim + (w[j] - pairs) * V;
                        r0[j] = *(const uint4*)(src[j] + d);
                        if (w[j] < pairs) r1[j] = *(const uint4*)(src[j] + d + half);
                    } else if (MODE != RM_SCALAR) {
                        r0[j] = *(const uint4*)(src[j] + w[j] * V);
                    }
                } else if (u < total) {
                    const int h = (u - coded) / vch, c = u - coded - h * vch;
                    w[j] = -1;
                    dst[j] = vrow + h * a.hs + c * V;
                    r0[j] = *(const uint4*)((const E*)a.v + i * a.v_stride + h * a.D + c * V);
                }
            }
            if (MODE != RM_NONE && !table) {
                __syncthreads();   // the previous token's table has been read
                for (int p = threadIdx.x; p < half; p += blockDim.x) cs[p] = phase(position, a.turns[p], a.m);
                __syncthreads();
                table = true;
            }
#pragma unroll
            for (int j = 0; j < AP_UNITS; ++j) {
                if (w[j] == -2) continue;
                if (w[j] == -1) {
                    *(uint4*)dst[j] = r0[j];
                } else if (MODE == RM_NONE) {
                    *(uint4*)(dst[j] + w[j] * V) = r0[j];
                } else if (MODE == RM_HALF) {
                    if (w[j] < pairs) {
                        float x1[V], x2[V], y1[V], y2[V];
                        Chunk<E>::unpack(r0[j], x1);
                        Chunk<E>::unpack(r1[j], x2);
                        const int d = w[j] * V;
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float2 t = cs[d + e];
                            y1[e] = x1[e] * t.x - x2[e] * t.y;
                            y2[e] = x2[e] * t.x + x1[e] * t.y;
                        }
                        *(uint4*)(dst[j] + d) = Chunk<E>::pack(y1);
                        *(uint4*)(dst[j] + d + half) = Chunk<E>::pack(y2);
                    } else {
                        *(uint4*)(dst[j] + a.dim + (w[j] - pairs) * V) = r0[j];
                    }
                } else if (MODE == RM_INTER) {
                    float x[V], y[V];
                    Chunk<E>::unpack(r0[j], x);
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const int p = (w[j] * V + e) / 2;
                        const bool in = p < half;
                        const float2 t = in ? cs[p] : make_float2(1.f, 0.f);
                        y[e] = in ? x[e] * t.x - x[e + 1] * t.y : x[e];
                        y[e + 1] = in ? x[e + 1] * t.x + x[e] * t.y : x[e + 1];
                    }
                    *(uint4*)(dst[j] + w[j] * V) = Chunk<E>::pack(y);
                } else {
                    if (w[j] < half) {
                        const float x1 = to_f(src[j][w[j]]), x2 = to_f(src[j][w[j] + half]);
                        const float2 t = cs[w[j]];
                        put(dst[j] + w[j], x1 * t.x - x2 * t.y);
                        put(dst[j] + w[j] + half, x2 * t.x + x1 * t.y);
                    } else {
                        dst[j][w[j] + half] = src[j][w[j] + half];
                    }
                }
            }
        }
    }
}

template <typename E>
jpi_status launch(const AppendArgs& a, int mode, cudaStream_t st) {
    constexpr int V = Chunk<E>::V;
    const int half = a.dim / 2;
    const int per = mode == RM_HALF ? half / V + (a.D - a.dim) / V : mode == RM_SCALAR ? a.D - half : a.D / V;
    const int total = (a.H + a.K) * per + (a.v ? a.K * (a.D / V) : 0);
    const int threads = total >= 512 ? 256 : total >= 256 ? 128 : total > 32 ? 64 : 32;
    const long long grid = a.n < (1 << 20) ? a.n : (1 << 20);
    switch (mode) {
        case RM_NONE: k_kv_append<E, RM_NONE><<<(unsigned)grid, threads, 0, st>>>(a); break;
        case RM_HALF: k_kv_append<E, RM_HALF><<<(unsigned)grid, threads, 0, st>>>(a); break;
        case RM_INTER: k_kv_append<E, RM_INTER><<<(unsigned)grid, threads, 0, st>>>(a); break;
        default: k_kv_append<E, RM_SCALAR><<<(unsigned)grid, threads, 0, st>>>(a); break;
    }
    JPI_CUDA_TRY(cudaGetLastError());
    return JPI_OK;
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
    a.tokens = tokens;
    a.n = (long long)batch * tokens;
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
    return h->bf16 ? launch<__nv_bfloat16>(a, mode, st) : launch<float>(a, mode, st);
}

}  // namespace jpi
