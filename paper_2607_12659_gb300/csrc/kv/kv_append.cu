// Rotary coding and cache write (jpi_kv_append).
//
// Pair i of a head, (x1, x2), turns by the angle a = position theta_i:
//   y1 = m (x1 cos a - x2 sin a),  y2 = m (x2 cos a + x1 sin a).
// The table holds theta_i / 2 pi, turns per position, as a fraction of 2^64, so that the phase
// position * turns is an integer product whose wrap-around is the reduction modulo a whole turn,
// without error of its own. The phase is off by the table's error times the position, less than |position| 2^-53 turns (an entry, at
// most 1 / 2 pi, comes of a power, a quotient or two and a division by 2 pi in 64-bit floating point: a few times 2^-53 of itself), and
// by 2^-26 where its 32 leading bits become an fp32 number of half turns in [-1, 1): a 32-bit angle would be off by
// whole turns far out. sincospif takes it from there. At position 131071 that is 2^-26 turns, at 2^31 up to 2^-22.
//
// Bound by memory: every element is read and written once. A block takes tokens in turn; a thread has the same
// units (a 16-byte chunk, or the two chunks of a half-layout pair) of each and copies them asynchronously into shared
// memory of its own, three tokens ahead, while a token's sines and cosines are computed, once for all heads, and shared.
// (With a block per token, 4 prompts of 2048 tokens of 8 heads of 256 took 21 us, a chain of three latencies in each block;
// with one token ahead in registers 23, too few bytes in flight.)

#include "kv_code.cuh"
#include "../ptx.h"

#include <algorithm>

namespace jpi {
namespace {

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

constexpr int AP_UNITS = 2;         // units of a thread
constexpr int AP_THREADS = 512;     // most of a block
constexpr int AP_STAGES = 4;        // tokens in hand
constexpr int AP_RUN = 64;          // tokens whose rows and positions are read together

template <typename E>
struct AppendUnit {
    int kind = -1;             // 0 query, 1 key, 2 value (copied), -1 none
    int w = 0;                 // chunk, pair of chunks or element of the head
    int at = 0;                // first element of its (first) chunk
    bool two = false;          // a second chunk, dim / 2 further on
    const E* src = nullptr;    // its head in token 0
    long long stride = 0;      // from one token to the next
    long long dst = 0;         // its head in the destination, without the token
};

template <typename E, int MODE>
__global__ void __launch_bounds__(AP_THREADS) k_kv_append(const __grid_constant__ AppendArgs a) {
    constexpr int V = Chunk<E>::V;
    extern __shared__ __align__(16) uint4 ap_stage[];   // [AP_STAGES][AP_UNITS][2][threads]
    __shared__ float2 table[2][AP_MAX_PAIRS + 8];   // (a last chunk may be part of one)
    __shared__ uint64_t turns[AP_MAX_PAIRS];
    __shared__ int2 token[AP_RUN];                      // (row, position)
    const int half = a.dim / 2, nth = blockDim.x, t = threadIdx.x;
    // Units of a coded head: its pairs, then what passes through; of a value head: its chunks.
    const int pairs = MODE == RM_HALF ? half / V : MODE == RM_SCALAR ? half : 0;
    const int per = MODE == RM_HALF ? pairs + (a.D - a.dim) / V : MODE == RM_SCALAR ? a.D - half : a.D / V;
    const int coded = (a.H + a.K) * per, vch = a.D / V, total = coded + (a.v ? a.K * vch : 0);
    if (MODE != RM_NONE)
        for (int p = t; p < half; p += nth) turns[p] = a.turns[p];
    const uint32_t mine = ptx::smem_u32(ap_stage) + 16 * t;
    // Where the table holds pair p: pair p mod PC of every chunk side by side, since the lanes of a warp read the same pair
    // of consecutive chunks (pair by pair they would meet in two banks: the 2048-token prompts took 24 us instead of 17).
    constexpr int PC = MODE == RM_HALF ? V : MODE == RM_INTER ? V / 2 : 1;   // pairs of a chunk
    const int chunks = (half + PC - 1) / PC;
    auto entry = [&](int p) { return p % PC * chunks + p / PC; };
    auto slot = [&](int stage, int j, int c) { return ((stage * AP_UNITS + j) * 2 + c) * nth; };
    const int step = gridDim.x;
    int turn = 0;
    for (int u0 = 0; u0 < total; u0 += AP_UNITS * nth) {
        AppendUnit<E> un[AP_UNITS];
#pragma unroll
        for (int j = 0; j < AP_UNITS; ++j) {
            const int u = u0 + j * nth + t;
            AppendUnit<E>& x = un[j];
            if (u < coded) {
                const int h = u / per;
                x.kind = h < a.H ? 0 : 1;
                x.w = u - h * per;
                x.src = h < a.H ? (const E*)a.q + h * a.D : (const E*)a.k + (h - a.H) * a.D;
                x.dst = h < a.H ? h * a.D : (h - a.H) * a.hs;
                x.stride = h < a.H ? a.q_stride : a.k_stride;
                x.two = MODE == RM_HALF && x.w < pairs;
                x.at = MODE == RM_HALF && !x.two ? a.dim + (x.w - pairs) * V : x.w * V;
            } else if (u < total) {
                const int h = (u - coded) / vch;
                x.kind = 2;
                x.w = u - coded - h * vch;
                x.src = (const E*)a.v + h * a.D;
                x.dst = h * a.hs;
                x.stride = a.v_stride;
                x.at = x.w * V;
            }
        }
        for (long long i0 = blockIdx.x; i0 < a.n; i0 += (long long)AP_RUN * step) {
            // Rows and positions of the next tokens i0, + step, ..
            __syncthreads();   // the last ones, and the tables, have been read
            const int count = (int)min((long long)AP_RUN, (a.n - i0 + step - 1) / step);
            for (int k = t; k < count; k += nth) token[k] = make_int2(a.row[i0 + (long long)k * step], a.position[i0 + (long long)k * step]);
            __syncthreads();
            auto live = [&](int k) { return token[k].x >= 0 && token[k].x < a.rows; };   // else padding
            auto fetch = [&](int k) {
                if (k < count && live(k)) {
                    const long long i = i0 + (long long)k * step;
#pragma unroll
                    for (int j = 0; j < AP_UNITS; ++j) {
                        const AppendUnit<E>& x = un[j];
                        if (x.kind < 0 || (MODE == RM_SCALAR && x.kind != 2)) continue;
                        const E* p = x.src + i * x.stride + x.at;
                        ptx::cp_async_16(mine + 16 * slot(k % AP_STAGES, j, 0), p, true);
                        if (x.two) ptx::cp_async_16(mine + 16 * slot(k % AP_STAGES, j, 1), p + half, true);
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
#pragma unroll
            for (int k = 0; k < AP_STAGES - 1; ++k) fetch(k);
            for (int k = 0; k < count; ++k) {
                fetch(k + AP_STAGES - 1);
                if (!live(k)) continue;   // (the same for the whole block)
                turn ^= 1;
                float2* cs = table[turn];   // the other may still be read; this one's readers are past the last barrier
                if (MODE != RM_NONE) {
                    for (int p = t; p < half; p += nth) cs[entry(p)] = phase(token[k].y, turns[p], a.m);
                    __syncthreads();
                }
                asm volatile("cp.async.wait_group %0;" ::"n"(AP_STAGES - 1) : "memory");
                const long long i = i0 + (long long)k * step;
                const long long row = (long long)a.by_tokens.div((uint32_t)i) * a.cs + token[k].x * a.rs;
#pragma unroll
                for (int j = 0; j < AP_UNITS; ++j) {
                    const AppendUnit<E>& x = un[j];
                    if (x.kind < 0) continue;
                    E* dst = x.kind == 0 ? (E*)a.q_out + i * a.H * a.D + x.dst : (x.kind == 1 ? (E*)a.ck : (E*)a.cv) + row + x.dst;
                    if (MODE == RM_SCALAR && x.kind != 2) {
                        const E* src = x.src + i * x.stride;
                        if (x.w < half) {
                            const float x1 = to_f(src[x.w]), x2 = to_f(src[x.w + half]);
                            const float2 c = cs[entry(x.w)];
                            put(dst + x.w, x1 * c.x - x2 * c.y);
                            put(dst + x.w + half, x2 * c.x + x1 * c.y);
                        } else {
                            dst[x.w + half] = src[x.w + half];
                        }
                        continue;
                    }
                    const uint4 c0 = ap_stage[slot(k % AP_STAGES, j, 0) + t];
                    if (x.two) {
                        float x1[V], x2[V], y1[V], y2[V];
                        Chunk<E>::unpack(c0, x1);
                        Chunk<E>::unpack(ap_stage[slot(k % AP_STAGES, j, 1) + t], x2);
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float2 c = cs[e * chunks + x.w];
                            y1[e] = x1[e] * c.x - x2[e] * c.y;
                            y2[e] = x2[e] * c.x + x1[e] * c.y;
                        }
                        *(uint4*)(dst + x.at) = Chunk<E>::pack(y1);
                        *(uint4*)(dst + x.at + half) = Chunk<E>::pack(y2);
                    } else if (MODE == RM_INTER && x.kind != 2) {
                        float v[V], y[V];
                        Chunk<E>::unpack(c0, v);
#pragma unroll
                        for (int e = 0; e < V; e += 2) {
                            const int p = (x.at + e) / 2;
                            const bool in = p < half;
                            const float2 c = in ? cs[entry(p)] : make_float2(1.f, 0.f);
                            y[e] = in ? v[e] * c.x - v[e + 1] * c.y : v[e];
                            y[e + 1] = in ? v[e + 1] * c.x + v[e] * c.y : v[e + 1];
                        }
                        *(uint4*)(dst + x.at) = Chunk<E>::pack(y);
                    } else {
                        *(uint4*)(dst + x.at) = c0;
                    }
                }
            }
        }
        ptx::cp_async_wait_all();   // (empty groups)
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
    const size_t smem = (size_t)AP_STAGES * AP_UNITS * 2 * threads * 16;
    // Blocks that are resident together, by shared memory (to 150 KB of an SM) and threads.
    const long long most = (long long)num_sms * std::max<long long>(1, std::min<long long>(1536 / threads, (150 << 10) / (long long)(smem + 4096)));
    return kv_start(mode == RM_NONE ? k_kv_append<E, RM_NONE>
                                    : mode == RM_HALF ? k_kv_append<E, RM_HALF>
                                                      : mode == RM_INTER ? k_kv_append<E, RM_INTER> : k_kv_append<E, RM_SCALAR>,
                    (long long)std::min<long long>(a.n, most), threads, smem, false, st, a);
}

}  // namespace

jpi_status kv_append_prepare() {
    const int most = AP_STAGES * AP_UNITS * 2 * AP_THREADS * 16;
    auto set = [&](const void* f) { return cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, most); };
    JPI_CUDA_TRY(set((const void*)k_kv_append<float, RM_NONE>));
    JPI_CUDA_TRY(set((const void*)k_kv_append<float, RM_HALF>));
    JPI_CUDA_TRY(set((const void*)k_kv_append<float, RM_INTER>));
    JPI_CUDA_TRY(set((const void*)k_kv_append<float, RM_SCALAR>));
    JPI_CUDA_TRY(set((const void*)k_kv_append<__nv_bfloat16, RM_NONE>));
    JPI_CUDA_TRY(set((const void*)k_kv_append<__nv_bfloat16, RM_HALF>));
    JPI_CUDA_TRY(set((const void*)k_kv_append<__nv_bfloat16, RM_INTER>));
    JPI_CUDA_TRY(set((const void*)k_kv_append<__nv_bfloat16, RM_SCALAR>));
    return JPI_OK;
}

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
