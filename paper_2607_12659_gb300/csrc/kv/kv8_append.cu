// New tokens into a cache held in 8 bits (jpi_kv8_append).
//
// An element x of a block of rows and head is held as the e4m3 code of x / s, s = 2^(e - 127) the least power of two with
// max |x| <= 448 s over the block's elements: division by s is exact, so a code is one rounding of fp32 x, and a scale that
// grows as rows come moves the codes before by a power of two, which e4m3 holds exactly but for its subnormals. (A scale that is
// the maximum itself would round every code of the block again at each step.)
//
// Bound by memory. A team of warps has one KV head's keys or values in one block of rows: the new rows' loads are on
// their way together, held by groups of lanes (kv_heads.cuh), which normalise and turn them in registers; the maximum is
// joined over the team, and the codes are written from the same registers. A (row, pair) has one user here, so its sine
// and cosine need no table. The queries' tokens are blocks of the same launch.

#include "kv8.cuh"
#include "kv_heads.cuh"

namespace jpi {
namespace {

struct Append8Args {
    HeadArgs h;               // (its H queries; K of them are none of its tokens' blocks')
    CodeTokens ct;            // of the queries
    int K;
    const int *start, *count;
    uint8_t *ck, *cv, *ks, *vs;
    long long cs, rs, hs;
    int rows, n_log2, nblk;   // rows of a cache, of a block (log2), blocks of a cache
    int touch;                // blocks that a request's tokens can touch
    int team, teams;          // warps of a unit, units of a block
    uint32_t units, blocks;   // of keys and values; the queries' blocks follow
    KvDiv by_touch, by_K;
};

// Rows [first, end) of cache b that the call writes.
__device__ __forceinline__ int2 new_rows(const Append8Args& a, int b) {
    const int s = a.start[b], c = a.count ? min(max(a.count[b], 0), a.h.tokens) : a.h.tokens;
    if (s < 0 || s >= a.rows) return make_int2(0, 0);
    return make_int2(s, min(s + c, a.rows));
}

// One team of warps' unit: the keys or the values of one KV head in one block of rows. The team's threads meet at barrier
// `bar` (a single warp: nowhere).
template <typename E, int MODE>
__device__ __forceinline__ void store8(const Append8Args& a, uint32_t unit, int team, float* most) {
    constexpr int V = Chunk<E>::V;
    constexpr int PASSES = V == 8 ? 4 : 8;   // rows of a group of lanes
    uint32_t j, kvh;
    const bool value = unit & 1;
    const int b = (int)a.by_K.div(a.by_touch.div(unit >> 1, j), kvh);
    const int2 span = new_rows(a, b);
    const int first = ((span.x >> a.n_log2) + (int)j) << a.n_log2, lo = max(first, span.x), hi = min(first + (1 << a.n_log2), span.y);
    if (lo >= hi) return;
    const int size = a.team * 32, t = threadIdx.x - team * size, groups = size >> a.h.lanes_log2, grp = t >> a.h.lanes_log2;
    const HeadLane<E, MODE> ln(t & ((1 << a.h.lanes_log2) - 1), a.h.D, a.h.dim);
    uint8_t* scale = (value ? a.vs : a.ks) + ((long long)b * a.K + kvh) * a.nblk + (first >> a.n_log2);
    uint8_t* codes = (value ? a.cv : a.ck) + b * a.cs + kvh * a.hs;
    const int e_old = first < span.x ? *scale : 0;
    const long long tok0 = (long long)b * a.h.tokens + (lo - span.x);
    const long long stride = value ? a.h.v_stride : a.h.k_stride;
    const E* src = static_cast<const E*>(value ? a.h.v : a.h.k) + tok0 * stride + kvh * a.h.D;
    uint4 raw[PASSES][2];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = p * groups + grp;
        ln.load(src + r * stride, lo + r < hi, raw[p]);
    }
    float2 x[PASSES][V];
    float top = 0.f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        if (lo + p * groups >= hi) break;   // (the same for the team)
        const int r = p * groups + grp;
        const bool in = lo + r < hi;
        if (value) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float z[V];
                Chunk<E>::unpack(raw[p][c], z);
#pragma unroll
                for (int i = 0; i < V / 2; ++i) x[p][c * (V / 2) + i] = make_float2(z[2 * i], z[2 * i + 1]);
            }
        } else {
            const int position = MODE != RM_NONE && in ? a.h.position[tok0 + r] : 0;
            constexpr int PC = pairs_of_chunk<E, MODE>();
            auto rot = [&](int q, float (&c)[PC], float (&s)[PC]) {
#pragma unroll
                for (int i = 0; i < PC; ++i) {
                    const int pr = q * PC + i;
                    const float2 z = phase_near(position, pr < a.h.dim / 2 ? a.h.turns[pr] : 0, a.h.m);
                    c[i] = z.x;
                    s[i] = z.y;
                }
            };
            const float* w = a.h.k_weight;
            auto weight = [&](int i) {
                const int c = 4 * i / V, d = ln.c[c] * V + 4 * i % V;
                return w && ln.live[c] ? make_float4(w[d], w[d + 1], w[d + 2], w[d + 3]) : make_float4(1.f, 1.f, 1.f, 1.f);
            };
            auto other = [&](int d) { return w ? w[d] : 1.f; };
            code_head<E, MODE>(ln, a.h, src + r * stride, in, raw[p], weight, other, rot, x[p]);
        }
        if (in) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float y = fabsf(x[p][i].x), z = fabsf(x[p][i].y);
                if (ln.live[i / (V / 2)] && y < INFINITY) top = fmaxf(top, y);
                if (ln.live[i / (V / 2)] && z < INFINITY) top = fmaxf(top, z);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (a.team > 1) {
        most += team * a.team;
        if ((t & 31) == 0) most[t >> 5] = top;
        ptx::named_bar_sync(1 + team, size);   // (and every thread has the old scale)
        for (int w = 0; w < a.team; ++w) top = fmaxf(top, most[w]);
    } else {
        __syncwarp();
    }
    const int e = max(kv8_exponent(top), e_old);
    const float inv = kv8_scale((uint32_t)max(254 - e, 0));   // (of a kept scale of 254 it is 2^-127, no normal number)
    if (t == 0) *scale = (uint8_t)e;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = lo + p * groups + grp;
        if (r >= hi) break;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (!ln.live[c]) continue;
            uint32_t w[V / 4];
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const float2 y = x[p][c * (V / 2) + 2 * i], z = x[p][c * (V / 2) + 2 * i + 1];
                w[i] = kv8_codes(y.x * inv, y.y * inv, z.x * inv, z.y * inv);
            }
            uint8_t* dst = codes + r * a.rs + ln.c[c] * V;
            if constexpr (V == 8)
                *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
            else
                *reinterpret_cast<uint32_t*>(dst) = w[0];
        }
    }
    if (first < span.x && e > e_old) {   // (a scale of 255 is above every other)
        const float f = kv8_pow2(127 + e_old - e);
        const int per = a.h.D / 16, n = (span.x - first) * per;
        for (int i = t; i < n; i += size) {
            uint4* at = reinterpret_cast<uint4*>(codes + (first + i / per) * a.rs + i % per * 16);
            uint4 u = *at;
            uint32_t* w = &u.x;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float z[4];
                kv8_values(w[k], z);
                w[k] = kv8_codes(z[0] * f, z[1] * f, z[2] * f, z[3] * f);
            }
            *at = u;
        }
    }
}

template <typename E, int MODE>
__global__ void __launch_bounds__(CT_THREADS) k_kv8_append(const __grid_constant__ Append8Args a) {
    __shared__ CodeWeights weights;
    __shared__ float most[CT_THREADS / 32];
    __shared__ __align__(16) CodeTable table[CT_THREADS / 32];
    if (blockIdx.x < a.blocks) {
        const int team = threadIdx.x / (32 * a.team);
        const uint32_t unit = blockIdx.x * a.teams + team;
        if (team < a.teams && unit < a.units) store8<E, MODE>(a, unit, team, most);
        return;
    }
    auto place = [&](int tok) {
        uint32_t t;
        const int2 span = new_rows(a, (int)a.h.by_tokens.div((uint32_t)tok, t));
        return (int)t < span.y - span.x ? 0 : -1;
    };
    auto at = [](long long, int) { return 0ll; };
    load_weights<E, MODE>(a.h, weights);
    __syncthreads();
    code_tokens<E, MODE>(a.h, a.ct, weights, table[threadIdx.x >> 5], (blockIdx.x - a.blocks) * (blockDim.x >> 5) + (threadIdx.x >> 5),
                         (gridDim.x - a.blocks) * (blockDim.x >> 5), static_cast<E*>(nullptr), static_cast<E*>(nullptr), 0, place, at);
}

template <typename E>
jpi_status launch(const Append8Args& a, int mode, unsigned blocks, int threads, cudaStream_t st) {
    return kv_start(mode == RM_NONE ? k_kv8_append<E, RM_NONE>
                                    : mode == RM_HALF ? k_kv8_append<E, RM_HALF>
                                                      : mode == RM_INTER ? k_kv8_append<E, RM_INTER> : k_kv8_append<E, RM_SCALAR>,
                    dim3(blocks), threads, 0, false, st, a);
}

}  // namespace

jpi_status launch_kv8_append(const jpi_kv_handle* h, const void* q, long long q_stride, const void* k, long long k_stride,
                             const void* v, long long v_stride, const jpi_kv_norm* norm, const int* position, const int* start,
                             const int* count, int batch, int tokens, void* q_out, const jpi_kv8_cache* cache, cudaStream_t st) {
    Append8Args a = {};
    a.h.q = q;
    a.h.k = k;
    a.h.v = v;
    a.h.q_stride = q_stride;
    a.h.k_stride = k_stride;
    a.h.v_stride = v_stride;
    a.h.position = position;
    a.h.q_out = q_out;
    a.h.H = q ? h->H : 0;
    a.h.batch = batch;
    a.h.tokens = tokens;
    a.h.norm = norm != nullptr;
    if (norm) {
        a.h.q_weight = norm->q_weight;
        a.h.k_weight = norm->k_weight;
        a.h.eps = norm->eps;
    }
    int threads = 128;
    const int mode = plan_code_tokens(h, a.h, a.ct, 0);
    a.K = h->K;
    a.start = start;
    a.count = count;
    a.rows = cache->rows;
    a.n_log2 = cache->block == 16 ? 4 : cache->block == 32 ? 5 : 6;
    a.nblk = (cache->rows + cache->block - 1) / cache->block;
    a.touch = 1;
    long long units = 0;
    if (k) {
        a.ck = static_cast<uint8_t*>(cache->k);
        a.cv = static_cast<uint8_t*>(cache->v);
        a.ks = cache->k_scale;
        a.vs = cache->v_scale;
        a.cs = cache->cache_stride;
        a.rs = cache->row_stride;
        a.hs = cache->head_stride;
        a.touch = (int)std::min<long long>(a.nblk, ((long long)tokens + 2 * cache->block - 2) / cache->block);
        units = 2ll * batch * h->K * a.touch;
        // Warps of a unit: two rows of its block for each group of lanes, as many more as that needs to fit its passes.
        const int rows = std::min(tokens, cache->block);
        a.team = 1;
        while (a.team < CT_THREADS / 32 && (a.team * 32 >> a.h.lanes_log2) * 2 < rows) a.team *= 2;
        threads = std::max(threads, a.team * 32);
        a.teams = threads / 32 / a.team;
        a.blocks = (uint32_t)((units + a.teams - 1) / a.teams);
    }
    a.by_touch = KvDiv((uint32_t)a.touch);
    a.by_K = KvDiv((uint32_t)h->K);
    if (units > 0x7fffffffll) {
        set_error("the call needs more than 2^31 blocks");
        return JPI_ERR_SHAPE;
    }
    a.units = (uint32_t)units;
    const unsigned blocks = a.blocks + (q ? code_blocks(h, a.ct, threads, 512 / threads) : 0);
    return h->bf16 ? launch<__nv_bfloat16>(a, mode, blocks, threads, st) : launch<float>(a, mode, blocks, threads, st);
}

}  // namespace jpi
