// Accumulated attention weight of cached keys (jpi_kv_weigh).
//
//   out[j] = decay in[j] + sum over rows r that see j of exp(s_rj - lse_r),  s_rj = scale q_r . k_j,
// with lse from jpi_kv_attend, so that no maximum has to be found and keys are independent of each other.
// A key's sum is formed by one block in a fixed order and written once: no atomics, no partial results in
// global memory.
//
// bf16: a warp keeps 16 keys in registers as the rows of mma.sync and streams the query rows past them, 8 at
// a time (the sum over d may run in any order, so lane (g, j) takes 16-byte chunk 4 i + j of its key and of its query
// row as the four element pairs of two k-steps: both come from global memory as they lie); a lane adds up the weights of
// its two keys, and the four lanes of a key and the warps that share it are joined at the end. Small calls are latency:
// 6 to 8 us a call, two of them the launch; larger ones go to the tensor-core tiles (kv_weigh_t5.cu). fp32 on CUDA
// cores: a key per lane.

#include "kv_rows.cuh"
#include "kv_weigh.h"

#include <algorithm>

namespace jpi {
namespace {

constexpr int WG_WARPS = 8;
constexpr int WG_THREADS = 32 * WG_WARPS;

struct WeighArgs {
    KvCall c;
    const float* lse;
    float decay;
    const float *pin, *oin;
    float *pout, *oout;
    int wr_p, wr_o;              // warps of a block that share its keys, each with every wr-th row tile
    int tiles_p, tiles_o;        // key blocks per cache and head
    long long blocks_p;
};

struct KeyPiece {
    bool prefix;
    int cache, kvh, tile, wr;
    RowTile t;
};
__device__ __forceinline__ KeyPiece key_piece(const WeighArgs& a) {
    KeyPiece x;
    long long i = blockIdx.x;
    x.prefix = i < a.blocks_p;
    if (!x.prefix) i -= a.blocks_p;
    const int tiles = x.prefix ? a.tiles_p : a.tiles_o;
    x.wr = x.prefix ? a.wr_p : a.wr_o;
    x.tile = (int)(i % tiles);
    i /= tiles;
    x.kvh = (int)(i % a.c.K);
    x.cache = (int)(i / a.c.K);
    const int toks = x.prefix ? a.c.batch / a.c.groups * a.c.tokens : a.c.tokens;
    x.t.tok0 = (long long)x.cache * toks;
    x.t.head0 = x.kvh * a.c.gq;
    x.t.R = toks * a.c.gq;
    x.t.r0 = 0;
    return x;
}
// Rows of the piece's cache that hold keys: the prefix's length, or the most that a token of the request sees.
__device__ __forceinline__ int live_keys(const WeighArgs& a, const KeyPiece& x, int* shared) {
    const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
    if (x.prefix) return min(max(s.len[x.cache], 0), s.rows);
    if (threadIdx.x == 0) *shared = 0;
    __syncthreads();
    int n = 0;
    for (int t = threadIdx.x; t < a.c.tokens; t += WG_THREADS) n = max(n, s.len[x.t.tok0 + t]);
    n = __reduce_max_sync(0xffffffffu, n);
    if ((threadIdx.x & 31) == 0) atomicMax(shared, n);
    __syncthreads();
    return min(*shared, s.rows);
}
__device__ __forceinline__ void write_weight(const WeighArgs& a, const KeyPiece& x, int key, float sum) {
    const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
    const float* in = x.prefix ? a.pin : a.oin;
    float* out = x.prefix ? a.pout : a.oout;
    const long long i = ((long long)x.cache * a.c.K + x.kvh) * s.rows + key;
    out[i] = in && a.decay != 0.f ? fmaf(a.decay, in[i], sum) : sum;
}

template <int DP>
__global__ void __launch_bounds__(WG_THREADS) k_kv_weigh_mma(const __grid_constant__ WeighArgs a) {
    __shared__ float part[WG_WARPS][16];
    __shared__ int top;
    constexpr int NC = DP / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
    ptx::grid_dep_launch();
    const KeyPiece x = key_piece(a);
    const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
    const int live = live_keys(a, x, &top);
    const int kt = WG_WARPS / x.wr, key0 = (x.tile * kt + warp / x.wr) * 16, wrow = warp % x.wr;
    float acc0 = 0.f, acc1 = 0.f;   // keys g and g + 8
    if (key0 < live) {
        uint4 kf[NC][2];
        const __nv_bfloat16* kp = (const __nv_bfloat16*)s.k + x.cache * s.cs + x.kvh * s.hs + (long long)(key0 + g) * s.rs + 8 * j;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const bool in = 8 * (4 * i + j) < a.c.D;
            kf[i][0] = kr_ld(kp + 32 * i, in && key0 + g < live);
            kf[i][1] = kr_ld(kp + 8 * s.rs + 32 * i, in && key0 + g + 8 < live);
        }
        // A row tile's loads: its query rows, and of rows 2 j and 2 j + 1 the lse and what they see.
        struct Rows {
            uint4 q[NC];
            float ls[2];
            int n[2];
        };
        auto load = [&](int rt) {
            Rows y;
            const int rq = rt + g;
            const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.c.q) + 8 * j;
            if (rq < x.t.R) q += row_query(a.c, x.t, rq);
#pragma unroll
            for (int i = 0; i < NC; ++i) y.q[i] = kr_ld(q + 32 * i, rq < x.t.R && 8 * (4 * i + j) < a.c.D);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = rt + 2 * j + e;
                y.ls[e] = r < x.t.R ? a.lse[row_index(a.c, x.t, r)] : -INFINITY;
                y.n[e] = row_seen(a.c, x.prefix, x.cache, x.t, r);
            }
            return y;
        };
        const int step = x.wr * KR_ROWS;
        for (int rt = wrow * KR_ROWS; rt < x.t.R; rt += step) {
            const Rows y = load(rt);
            float sc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                kr_mma(sc, kf[i][0].x, kf[i][1].x, kf[i][0].y, kf[i][1].y, y.q[i].x, y.q[i].y);
                kr_mma(sc, kf[i][0].z, kf[i][1].z, kf[i][0].w, kf[i][1].w, y.q[i].z, y.q[i].w);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (y.ls[e] == -INFINITY) continue;
                if (key0 + g < y.n[e]) acc0 += kr_ex2(fmaf(sc[e], a.c.scale, -y.ls[e]) * KR_LOG2E);
                if (key0 + g + 8 < y.n[e]) acc1 += kr_ex2(fmaf(sc[2 + e], a.c.scale, -y.ls[e]) * KR_LOG2E);
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        acc0 += __shfl_xor_sync(0xffffffffu, acc0, o);
        acc1 += __shfl_xor_sync(0xffffffffu, acc1, o);
    }
    if (j == 0) {
        part[warp][g] = acc0;
        part[warp][g + 8] = acc1;
    }
    __syncthreads();
    if (wrow == 0 && lane < 16 && key0 + lane < live) {
        float sum = part[warp][lane];
        for (int i = 1; i < x.wr; ++i) sum += part[warp + i][lane];
        write_weight(a, x, key0 + lane, sum);
    }
}

// A warp takes 32 keys, one a lane, and 8 query rows at a time; 32 elements of both pass through its shared memory, loaded in
// whole lines a step ahead. (Bound by the reads of shared memory, 9 for 32 fused products, and latency: 2 requests of 34 tokens of 8
// heads of 256 over 62 keys took 68 us with each lane reading its key from memory, 32 sectors a load, and 44 so; 12 requests
// of 7 tokens of 8 heads of 128 over 26 keys 18.5, with the rows read from memory too, and 11.)
__global__ void __launch_bounds__(WG_THREADS) k_kv_weigh_f32(const __grid_constant__ WeighArgs a) {
    constexpr int CH = 8;   // 16-byte pieces of a row in a step
    __shared__ float4 rows[WG_WARPS][KR_ROWS][CH];
    __shared__ float4 kbuf[WG_WARPS][32][CH + 1];   // (the pad spreads the lanes' rows over the banks)
    __shared__ float part[WG_WARPS][32];
    __shared__ int top;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = a.c.D;
    ptx::grid_dep_launch();
    const KeyPiece x = key_piece(a);
    const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
    const int live = live_keys(a, x, &top);
    const int kt = WG_WARPS / x.wr, key0 = (x.tile * kt + warp / x.wr) * 32, key = key0 + lane, wrow = warp % x.wr;
    float acc = 0.f;
    if (key0 < live) {
        const int c = lane & 7, sub = lane >> 3;   // this lane's piece of a step, of every fourth row
        const float* kp = (const float*)s.k + x.cache * s.cs + x.kvh * s.hs + (long long)(key0 + sub) * s.rs + 4 * c;
        for (int rt = wrow * KR_ROWS; rt < x.t.R; rt += x.wr * KR_ROWS) {
            float p[KR_ROWS], ls[KR_ROWS];
            int n[KR_ROWS];
            const float* q[2];
            float4 k[8], v[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                q[j] = static_cast<const float*>(a.c.q) + row_query(a.c, x.t, min(rt + sub + 4 * j, x.t.R - 1)) + 4 * c;
            auto load = [&](int d0) {
                const bool in = d0 + 4 * c < D;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    k[j] = in && key0 + sub + 4 * j < live ? __ldg((const float4*)(kp + 4 * j * s.rs + d0)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int j = 0; j < 2; ++j) v[j] = in ? __ldg((const float4*)(q[j] + d0)) : make_float4(0.f, 0.f, 0.f, 0.f);
            };
            load(0);
#pragma unroll
            for (int r = 0; r < KR_ROWS; ++r) {
                p[r] = 0.f;
                ls[r] = a.lse[row_index(a.c, x.t, min(rt + r, x.t.R - 1))];
                n[r] = row_seen(a.c, x.prefix, x.cache, x.t, rt + r);
            }
#pragma unroll 1
            for (int d0 = 0; d0 < D; d0 += 4 * CH) {
                __syncwarp();   // the step before has been read
#pragma unroll
                for (int j = 0; j < 8; ++j) kbuf[warp][sub + 4 * j][c] = k[j];
#pragma unroll
                for (int j = 0; j < 2; ++j) rows[warp][sub + 4 * j][c] = v[j];
                __syncwarp();
                if (d0 + 4 * CH < D) load(d0 + 4 * CH);
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const float4 z = kbuf[warp][lane][i];
#pragma unroll
                    for (int r = 0; r < KR_ROWS; ++r) {
                        const float4 y = rows[warp][r][i];
                        p[r] = fmaf(y.x, z.x, fmaf(y.y, z.y, fmaf(y.z, z.z, fmaf(y.w, z.w, p[r]))));
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < KR_ROWS; ++r)
                if (key < n[r] && ls[r] != -INFINITY) acc += expf(fmaf(p[r], a.c.scale, -ls[r]));
        }
    }
    part[warp][lane] = acc;
    __syncthreads();
    if (wrow == 0 && key < live) {
        float sum = acc;
        for (int i = 1; i < x.wr; ++i) sum += part[warp + i][lane];
        write_weight(a, x, key, sum);
    }
}

// Warps that share a block's keys: as many as leave every SM a block, and each warp a row tile.
int row_warps(const jpi_kv_handle* h, const KvCall& c, bool prefix, int keys, int* tiles) {
    const KvSide& s = prefix ? c.prefix : c.own;
    const long long R = (long long)(prefix ? c.batch / c.groups : 1) * c.tokens * c.gq;
    const long long caches = (long long)(prefix ? c.groups : c.batch) * c.K, rt = (R + KR_ROWS - 1) / KR_ROWS;
    int wr = 1;
    auto count = [&](int w) { return (s.rows + keys * (WG_WARPS / w) - 1) / (keys * (WG_WARPS / w)); };
    while (wr < WG_WARPS && wr * 2 <= rt && caches * count(wr) < h->num_sms) wr *= 2;
    *tiles = s.rows ? count(wr) : 0;
    return wr;
}

}  // namespace

jpi_status launch_kv_weigh(jpi_kv_handle* h, const KvCall& c, const float* lse, float decay, const float* prefix_in,
                           float* prefix_out, const float* own_in, float* own_out, cudaStream_t st) {
    WeighArgs a;
    a.c = c;
    a.lse = lse;
    a.decay = decay;
    a.pin = prefix_in;
    a.oin = own_in;
    a.pout = prefix_out;
    a.oout = own_out;
    const int keys = h->bf16 ? 16 : 32;
    a.wr_p = row_warps(h, c, true, keys, &a.tiles_p);
    a.wr_o = row_warps(h, c, false, keys, &a.tiles_o);
    // Many rows on one prefix go to the tensor-core tiles.
    const bool tiles = kv_weigh_tiles(h, c);
    a.blocks_p = tiles ? 0 : (long long)c.groups * c.K * a.tiles_p;
    const long long blocks = a.blocks_p + (long long)c.batch * c.K * a.tiles_o;
    if (blocks > 0x7fffffffll) {
        set_error("the call needs more than 2^31 blocks");
        return JPI_ERR_SHAPE;
    }
    if (blocks > 0)
        JPI_TRY(kv_start(!h->bf16 ? k_kv_weigh_f32
                                  : h->D <= 64 ? k_kv_weigh_mma<64> : h->D <= 128 ? k_kv_weigh_mma<128> : k_kv_weigh_mma<256>,
                         blocks, WG_THREADS, 0, false, st, a));
    if (tiles) return launch_kv_weigh_t5(h, c, lse, decay, prefix_in, prefix_out, blocks > 0 && h->pdl, st);
    return JPI_OK;
}

}  // namespace jpi
