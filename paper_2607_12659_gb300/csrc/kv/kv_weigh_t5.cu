// The prefix side of jpi_kv_weigh on tcgen05: 128 keys a block, all query rows of the run past them in tiles of
// 128. Keys are the rows of the products (TMEM lanes) and query rows their columns, so that a key's weights
// are one lane's: no maximum, no exchange between lanes until the end, nothing to mask (a row past the prefix's end is
// a lane that is not written), and a sum's order is fixed.
//   warp 0      one thread: the key tile by bulk tensor copies, once
//   warp 1      one thread: S = K Q^T (M = 128, N = 128, K = D) into one of two TMEM buffers
//   warps 2-9   query rows gathered into one of two shared-memory tiles (128-byte swizzle) by asynchronous copies,
//               with their -lse: four warps fill each tile, so that one's copies fly while the other's are issued
//   warps 10-17 two threads per key (its TMEM lane), half of a tile's columns each: the sum of exp(scale s - lse)
// Bound by 2^x and the products alike (128 x R of the one, 4096 cycles of the other at R = 512, D = 256); the keys come
// from memory once and the query rows from L2 once per 128 keys. Every wait is bounded; where one gave up, in any block that shares the
// keys, their weights stay as they were.

#include "kv_rows.cuh"
#include "kv_maps.h"
#include "kv_weigh.h"

namespace jpi {
namespace {

constexpr int WT_KEYS = 128, WT_ROWS = 128;
constexpr int WT_LOAD = 128, WT_SUM = 256;          // threads that load a tile, and of the sums
constexpr int WT_THREADS = 64 + 2 * WT_LOAD + WT_SUM;
constexpr uint64_t WT_WAIT_NS = 200ull * 1000 * 1000;

struct WeighT5Args {
    KvCall c;
    const float* lse;
    float decay;
    const float* in;
    float* out;
    int tiles;           // key tiles per run and KV head
    int3 at;             // of the map's outer dimensions: heads, rows, runs
    int* err;
    KvDiv by_tiles, by_ranks;
    int ranks;           // blocks (a cluster) that share a key tile, each with every ranks-th row tile
};

template <int DP>
struct WtSmem {
    static constexpr int KBYTES = WT_KEYS * DP * 2, QBYTES = WT_ROWS * DP * 2;
    static constexpr int Q_OFF = KBYTES;                      // two tiles
    static constexpr int LSE_OFF = Q_OFF + 2 * QBYTES;        // [2][128] -lse
    static constexpr int SUM_OFF = LSE_OFF + 2 * WT_ROWS * 4; // [128] the second halves' sums
    static constexpr int BAR_OFF = SUM_OFF + WT_KEYS * 4;
    static constexpr int BYTES = BAR_OFF + 9 * 8 + 8;
    static_assert(BYTES <= 227 * 1024, "fits an SM");
    static constexpr uint32_t TMEM_COLS = 256;
};

template <int DP>
__global__ void __launch_bounds__(WT_THREADS, 1) k_kv_weigh_t5(const __grid_constant__ CUtensorMap kmap,
                                                               const __grid_constant__ WeighT5Args a) {
    using L = WtSmem<DP>;
    constexpr int NDB = DP / 64;
    constexpr uint32_t IDESC = ptx::idesc_bf16_f32(WT_KEYS, WT_ROWS);
    extern __shared__ __align__(1024) uint8_t wt_smem[];
    float* nlse = (float*)(wt_smem + L::LSE_OFF);
    float* sums = (float*)(wt_smem + L::SUM_OFF);
    uint64_t* kfull = (uint64_t*)(wt_smem + L::BAR_OFF);
    uint64_t* qfull = kfull + 1;     // 2: query tile in shared memory
    uint64_t* qempty = kfull + 3;    // 2: its products are done
    uint64_t* sfull = kfull + 5;     // 2: scores ready
    uint64_t* sfree = kfull + 7;     // 2: scores read
    uint32_t* tmem_slot = (uint32_t*)(kfull + 9);
    int* flag = (int*)(tmem_slot + 1);
    const int tid = threadIdx.x, warp = ptx::warp_index(), lane = tid & 31;
    uint32_t tile, kvh, rank;
    const int run = (int)a.c.by_K.div(a.by_tiles.div(a.by_ranks.div(blockIdx.x, rank), tile), kvh);
    const int len = min(max(a.c.prefix.len[run], 0), a.c.prefix.rows), key0 = (int)tile * WT_KEYS;
    if (key0 >= len) {
        ptx::grid_dep_wait();   // (ends after the kernel that started before it)
        return;
    }
    RowTile t;
    const int toks = a.c.batch / a.c.groups * a.c.tokens;
    t.tok0 = (long long)run * toks;
    t.head0 = (int)kvh * a.c.gq;
    t.R = toks * a.c.gq;
    t.r0 = 0;
    // Row tiles of this block: rank, rank + ranks, ..
    const int nt = ((t.R + WT_ROWS - 1) / WT_ROWS - (int)rank + a.ranks - 1) / a.ranks;

    if (warp == 0 && ptx::elect_one()) {
        ptx::prefetch_tmap(&kmap);
        ptx::mbar_init(kfull, 1);
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(&qfull[b], WT_LOAD);
            ptx::mbar_init(&qempty[b], 1);
            ptx::mbar_init(&sfull[b], 1);
            ptx::mbar_init(&sfree[b], WT_SUM);
        }
        ptx::fence_mbar_init();
        *flag = 0;
        ptx::mbar_expect_tx(kfull, (uint32_t)L::KBYTES);
        for (int db = 0; db < NDB; ++db)
            kv_load_box(wt_smem + db * (WT_KEYS * 128), &kmap, kfull, db * 64, a.at, (int)kvh, key0, run);
    }
    if (warp == 1) {
        ptx::tmem_alloc(tmem_slot, L::TMEM_COLS);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        // (the key tile is waited for below, also where a wait gave up: nothing may land after the block)
        if (lane == 0 && !ptx::mbar_wait_bounded(kfull, 0, WT_WAIT_NS)) *flag = DEV_TIMEOUT_WEIGHTS;
    } else if (warp == 1) {
        if (ptx::elect_one()) {
            const uint32_t kb = ptx::smem_u32(wt_smem), qb = kb + L::Q_OFF;
            bool good = ptx::mbar_wait_bounded(kfull, 0, WT_WAIT_NS);
            for (int i = 0; i < nt; ++i) {
                const int b = i & 1;
                if (good) good = ptx::mbar_wait_bounded(&qfull[b], (i >> 1) & 1, WT_WAIT_NS);
                if (i >= 2 && good) good = ptx::mbar_wait_bounded(&sfree[b], ((i >> 1) - 1) & 1, WT_WAIT_NS);
                ptx::tc_fence_after();
                if (good) {
                    const uint64_t kd = ptx::desc_sw128(kb), qd = ptx::desc_sw128(qb + (uint32_t)(b * L::QBYTES));
#pragma unroll
                    for (int db = 0; db < NDB; ++db)
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            ptx::mma_bf16(tmem + (uint32_t)(WT_ROWS * b), ptx::desc_add(kd, db * (WT_KEYS * 128) + kk * 32),
                                          ptx::desc_add(qd, db * (WT_ROWS * 128) + kk * 32), IDESC, (db | kk) != 0);
                }
                if (i + 2 < nt) ptx::mma_commit(&qempty[b]);
                ptx::mma_commit(&sfull[b]);
            }
            if (!good) *flag = DEV_TIMEOUT_MMA;
        }
    } else if (warp < 10) {
        const int b = (warp - 2) >> 2, lt = (tid - 64) % WT_LOAD;   // fills tile buffer b: tiles b, b + 2, ..
        bool good = true;
        constexpr int CH = DP / 8, RPI = WT_LOAD / CH;   // chunks of a row, rows of one pass of the loaders
        const int ch = lt % CH, rr0 = lt / CH;
        const bool dlive = 8 * ch < a.c.D;
        uint32_t hd_step;
        const uint32_t tok_step = a.c.by_gq.div((uint32_t)RPI, hd_step), gq = (uint32_t)a.c.gq;
        const __nv_bfloat16* base = static_cast<const __nv_bfloat16*>(a.c.q) + t.tok0 * a.c.q_stride +
                                    (long long)t.head0 * a.c.D + (dlive ? 8 * ch : 0);
        const uint32_t dst = ptx::smem_u32(wt_smem) + L::Q_OFF + b * L::QBYTES + (ch >> 3) * (WT_ROWS * 128);
        for (int i = b; i < nt; i += 2) {
            const int rt = ((int)rank + i * a.ranks) * WT_ROWS, rl = rt + lt;
            const float ls = rl < t.R ? a.lse[row_index(a.c, t, rl)] : -INFINITY;
            // Rows rt + rr0, + RPI, ..: token and head, stepped without a division. Past the run's rows nothing is read.
            int r = rt + rr0;
            uint32_t hd, tok = a.c.by_gq.div((uint32_t)r, hd);
            if (i >= 2 && good) good = ptx::mbar_wait_bounded(&qempty[b], ((i >> 1) - 1) & 1, WT_WAIT_NS);
#pragma unroll 8
            for (int rr = rr0; rr < WT_ROWS; rr += RPI) {
                const bool in = dlive && r < t.R;
                ptx::cp_async_16(dst + rr * 128 + (((ch & 7) ^ (rr & 7)) << 4),
                                 in ? base + (long long)tok * a.c.q_stride + hd * (uint32_t)a.c.D : base, in);
                r += RPI;
                tok += tok_step;
                hd += hd_step;
                if (hd >= gq) {
                    hd -= gq;
                    ++tok;
                }
            }
            if (i >= 2 && good) good = ptx::mbar_wait_bounded(&sfree[b], ((i >> 1) - 1) & 1, WT_WAIT_NS);   // the sums have read it
            nlse[b * WT_ROWS + lt] = ls == -INFINITY ? -INFINITY : -ls;   // a row that saw nothing gives nothing
            ptx::cp_async_wait_all();
            ptx::fence_proxy_async_smem();
            ptx::mbar_arrive(&qfull[b]);
        }
        if (!good) *flag = DEV_TIMEOUT_MMA;
    } else {
        const int key = (warp & 3) * 32 + lane, half = (warp - 10) >> 2;
        const uint32_t col0 = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(half * (WT_ROWS / 2));
        bool good = true;
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < nt; ++i) {
            const int b = i & 1;
            if (good) good = ptx::mbar_wait_bounded(&sfull[b], (i >> 1) & 1, WT_WAIT_NS);
            ptx::tc_fence_after();
            uint32_t s[4][16];
#pragma unroll
            for (int k = 0; k < 4; ++k) ptx::tmem_ld_x16(col0 + (uint32_t)(WT_ROWS * b + 16 * k), s[k]);
            ptx::tmem_ld_wait();
            const float4* nl = (const float4*)(nlse + b * WT_ROWS + half * (WT_ROWS / 2));
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const float4 n = nl[k];
                const uint32_t* x = s[k >> 2] + 4 * (k & 3);
                const float m[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float w = kr_ex2(fmaf(__uint_as_float(x[e]), a.c.scale, m[e]) * KR_LOG2E);
                    acc[e] += m[e] == -INFINITY ? 0.f : w;   // (whatever such a row's query holds)
                }
            }
            ptx::tc_fence_before();
            // Scores and -lse of this buffer are read: the next tile but one may take both.
            if (i + 2 < nt) ptx::mbar_arrive(&sfree[b]);
        }
        if (!good) *flag = DEV_TIMEOUT_MMA;
        const float sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
        if (half == 1) sums[key] = sum;
        ptx::named_bar_sync(1, WT_SUM);
        if (half == 0) sums[key] += sum;
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    // The sums of the blocks that share the keys, in their order.
    if (a.ranks > 1) ptx::cluster_sync_all();
    const int key = tid - (WT_THREADS - WT_SUM);
    if (rank == 0 && key >= 0 && key < WT_KEYS) {
        float w = sums[key];
        bool whole = *flag == 0;   // no block's rows are missing
        for (int k = 1; k < a.ranks; ++k) {
            w += ptx::dsmem_ld_f32(ptx::dsmem_map(ptx::smem_u32(sums + key), (uint32_t)k));
            whole = whole && __float_as_int(ptx::dsmem_ld_f32(ptx::dsmem_map(ptx::smem_u32(flag), (uint32_t)k))) == 0;
        }
        ptx::grid_dep_wait();   // the row kernel that started before this one: what follows this kernel has both
        if (key0 + key < len && whole) {
            const long long at = ((long long)run * a.c.K + kvh) * a.c.prefix.rows + key0 + key;
            a.out[at] = a.in && a.decay != 0.f ? fmaf(a.decay, a.in[at], w) : w;
        }
    }
    __syncwarp();
    if (a.ranks > 1) ptx::cluster_sync_all();   // (a block's shared memory lasts until its sums have been read)
    if (tid == 0 && *flag != 0) atomicCAS(a.err, 0, *flag);
    if (warp == 1) ptx::tmem_dealloc(tmem, L::TMEM_COLS);
}

template <int DP>
jpi_status launch_dim(const WeighT5Args& a, const CUtensorMap& map, bool early, cudaStream_t st) {
    return kv_start_clusters(k_kv_weigh_t5<DP>, (long long)a.tiles * a.c.K * a.c.groups * a.ranks, (unsigned)a.ranks, WT_THREADS,
                             WtSmem<DP>::BYTES, early, st, map, a);
}

}  // namespace

jpi_status kv_weigh_prepare(jpi_kv_handle* h) {
    if (!h->bf16 || h->D < 64) return JPI_OK;
    if (h->D <= 64)
        JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_weigh_t5<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, WtSmem<64>::BYTES));
    else if (h->D <= 128)
        JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_weigh_t5<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, WtSmem<128>::BYTES));
    else
        JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_weigh_t5<256>, cudaFuncAttributeMaxDynamicSharedMemorySize, WtSmem<256>::BYTES));
    return JPI_OK;
}

// The row kernel reads a key once for every 8 query rows, and its warps take those one after the other. Up to 16 M elements
// of keys read so it ends earlier, as long as the rows are not many: with 1 KV head at D = 256 and 16 own rows each,
// 128 rows over 1024, 4096 and 8192 keys take 5.3, 6.3 and 8.5 us there and 5.9, 6.0 and 6.1 here; 256 over 512 and 4096
// keys 6.8 and 8.7, here 7.1 and 7.2; 512 over 16 keys 9.5 and 7.0. Of fewer than 64 rows a tile is mostly empty: 32 rows over
// 16384 keys of 8 KV heads at D = 128 take 21 us there and 27 here.
bool kv_weigh_tiles(const jpi_kv_handle* h, const KvCall& c) {
    if (!h->bf16 || c.D < 64 || c.prefix.rows == 0) return false;
    KvMapDims m;
    const long long R = (long long)(c.batch / c.groups) * c.tokens * c.gq;
    const long long elements = (R + 7) / 8 * c.K * c.groups * c.prefix.rows * c.D;
    const bool take = h->tiles < 0 ? R >= 64 && (R >= 512 || elements > 16ll << 20) : h->tiles == 1;
    return take && kv_map_dims(c.prefix, c.K, c.D, c.groups, &m) &&
           (long long)((c.prefix.rows + WT_KEYS - 1) / WT_KEYS) * c.K * c.groups <= 0x7fffffffll / 8;
}

jpi_status launch_kv_weigh_t5(jpi_kv_handle* h, const KvCall& c, const float* lse, float decay, const float* in, float* out,
                              bool early, cudaStream_t st) {
    WeighT5Args a = {};
    a.c = c;
    a.lse = lse;
    a.decay = decay;
    a.in = in;
    a.out = out;
    a.tiles = (c.prefix.rows + WT_KEYS - 1) / WT_KEYS;
    a.by_tiles = KvDiv((uint32_t)a.tiles);
    a.err = h->dev_err;
    // Few keys and many rows: a row tile is 1.5 us of a block, one after the other, unless a cluster shares them. 1440
    // rows over 8 keys: 21 us by one block, 9 us by eight.
    const long long blocks = (long long)a.tiles * c.K * c.groups;
    const long long nt = ((long long)(c.batch / c.groups) * c.tokens * c.gq + WT_ROWS - 1) / WT_ROWS;
    a.ranks = 1;
    while (a.ranks < 8 && 2 * a.ranks <= nt && blocks * a.ranks * 2 <= h->num_sms) a.ranks *= 2;
    a.by_ranks = KvDiv((uint32_t)a.ranks);
    KvMapDims m;
    CUtensorMap map;
    if (!kv_map_dims(c.prefix, c.K, c.D, c.groups, &m) || !kv_make_map(m, c.prefix.k, c.D, WT_KEYS, &map)) {
        set_error("cuTensorMapEncodeTiled refused the prefix");
        return JPI_ERR_CUDA;
    }
    a.at = make_int3(m.at_head, m.at_row, m.at_cache);
    return c.D <= 64 ? launch_dim<64>(a, map, early, st) : c.D <= 128 ? launch_dim<128>(a, map, early, st) : launch_dim<256>(a, map, early, st);
}

}  // namespace jpi
