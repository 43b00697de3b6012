// Sides of jpi_kv_attend with many query rows on tcgen05: 128 query rows (tokens x heads of one KV head, of a run
// over its prefix or of a request over its own rows) per block over a range of their keys, in blocks of 64 keys. Where a
// request's query rows alone fill tiles, these take the prefix's keys and then the request's own in one pass, and a
// tile that is not split writes the result itself; else the run's rows share the prefix's tiles, and the parts are
// joined by k_kv_combine.
//   warp 0  one thread: K blocks by bulk tensor copies into a ring of NS slots (the first ones, of V too, before
//           the block has set itself up)
//   warp 1  one thread: V blocks into a ring of their own
//   warp 2  one thread: S_i = Q K_i^T (M = 128, N = 64, K = D) into one of two TMEM score buffers
//   warp 3  one thread: O += P_i V_i (M = 128, N = D, K = 64), V read as an MN-major operand
//   warps 4-  groups of eight: two threads per query row (its TMEM lane), half of a block's keys each: maximum, 2^x,
//           probabilities as bf16 back to tensor memory, over the scores they come from (the A operand of the
//           second product: no shared memory, and room on the SM for blocks of the row kernel). To D = 128 a block's
//           softmax takes twice as long as its products (1280 cycles for one group of warps, 610): two groups take the
//           even and the odd blocks, each with a maximum, sum and output of its own, joined at the end. At D = 256 the
//           products need that long, and tensor memory holds one output. O is rescaled only when a block's maximum passes the running one by
//           more than 8 in log2 units, so that probabilities stay below 2^8.
// The query rows are gathered by the softmax threads (tokens may lie at any stride and a row tile may begin and end
// inside a token's heads) into tensor memory as the A operand of the score products, which leaves all of shared memory
// to keys and values.
//
// Probabilities are rounded to bf16 once, each off by at most 2^-8 of itself, of either sign: with 128 rows a block there is
// no time for a second term as in the row kernel, which would be half as many products again, and the result's own rounding to
// bf16 is as large. The sum l takes them unrounded. A handle made with JPI_KV_TILES=0 does not come here.
//
// Rows past the last one that a query row of the tile sees may hold anything: their scores are replaced, and their
// values are cleared in shared memory before the product, since 0 times a NaN would reach every row. Own rows that
// only some of the query rows see are searched for infinities and NaN; a block that holds one is added row by row on
// CUDA cores instead (each row its own keys), and the product adds nothing.
//
// Each block leaves a part (unnormalised fp32 rows, (m, l)) for k_kv_combine, or the result: rows pass through shared
// memory (the ring, free by then) and leave by bulk copies, contiguous in global memory (about 27 bytes a cycle).
//
// Every wait is bounded; a wait that gives up records an error in the handle's word, and its thread waits for
// nothing more.

#include "kv_tiles.cuh"
#include "kv_attend.h"
#include "kv_maps.h"

#include <algorithm>

namespace jpi {
namespace {

constexpr int KP_ROWS = 128;
constexpr int KP_KEYS = 64;
constexpr int KP_SOFT = 256;   // threads of a softmax group
constexpr uint64_t KP_WAIT_NS = 200ull * 1000 * 1000;
constexpr float KP_RESCALE = 8.f;   // log2 units
// Query rows from which a side takes the tiles: 32, and of a prefix at D > 128, where a step of the row kernel is 16 keys
// only, as soon as that reads the keys twice. Microseconds of row kernel and tiles: 24 rows over 16384 and 65536 keys of
// 8 KV heads at D = 128 25.1 65.9 and 25.5 53.4, 32 rows 30.2 85.6 and 23.2 54.0; 16 rows over 32768 keys of one KV
// head at D = 256 19.4 and 14.0, 8 rows 14.9 and 14.1; 64 requests' own 2048 and 8192 rows at 8 query rows each 29.4
// 86.5 and 29.0 83.1.
constexpr int kp_least(bool own, int D) { return !own && D > 128 ? 9 : 32; }
// Elements of keys up to which a call stays with the row kernel, which reads a key once for every 8 query rows but has
// neither the tiles' long start nor their query rows to turn. Microseconds of row kernel and tiles where 16 own rows come with it:
// 1 KV head at D = 256, 256 rows over 64, 512, 1024 and 2048 keys (0.5, 4, 8 and 17 M elements): 8.2 11.3 11.8 17.4 and
// 11.8 12.5 12.6 14.0; 1024 rows over 256 and 512 keys (8 and 17 M): 11.6 17.9 and 13.5 13.4; 8 KV heads at D = 128, 128
// rows each over 512 and 1024 keys: 10.9 14.7 and 12.5 13.0; 512 rows at D = 64 over 2048 and 4096 keys: 10.7 15.2
// and 11.7 12.4.
constexpr long long KP_ROW_ELEMENTS = 10ll << 20;
constexpr int KP_FIXED = 5;         // start and end of a block, in key blocks

// Tiles of a run's rows over its prefix (0), or of a request's rows over its own keys (1), with `both` over the prefix's
// before them.
struct TileSide {
    int splits = 1, tiles = 0, part0 = 0;   // key ranges, row tiles per run or request and KV head, first part
    uint32_t blocks = 0;
    KvDiv by_splits, by_tiles;
};
struct TileMaps {
    CUtensorMap k[2], v[2];   // prefix, own
};
struct TileArgs {
    KvCall c;
    float c2;            // log2(e) * scale
    TileSide side[2];
    int3 at[2];          // of the maps' outer dimensions: heads, rows, caches
    bool both;
    KvDiv by_run;        // requests of a run
    float* po;           // [parts][rows][D]
    float2* pml;         // [rows][parts]
    long long rows;
    int parts;
    __nv_bfloat16* out;  // of a call of one part: the result, else null
    float* lse;
    int* err;
};

template <int DP>
struct KpSmem {
    static constexpr int NS = DP == 256 ? 2 : DP == 128 ? 3 : 4;
    static constexpr int KVBYTES = KP_KEYS * DP * 2;
    static constexpr int STAGE = 2 * KVBYTES;               // ring slot: K, then V
    static constexpr int OUT_LD = DP * 4 + 16;              // bytes of a staged output row: the pad spreads the banks
    static constexpr int RING = NS * STAGE > KP_ROWS * OUT_LD ? NS * STAGE : KP_ROWS * OUT_LD;
    static constexpr int NG = DP == 256 ? 1 : 2;            // softmax groups
    static constexpr int THREADS = 128 + NG * KP_SOFT;
    static constexpr int REGS = NG == 1 ? 96 : 72;          // the rest of the SM's is the row kernel's
    // Score buffers: a third where it fits, so that a group's next scores are there when it is through with the last
    // (with two they wait for the product that reads the probabilities lying over them).
    static constexpr int NB = DP == 256 ? 2 : 3;
    static constexpr int XM_OFF = RING;                     // [groups][2 blocks][2 key halves][128 rows]
    static constexpr int ML_OFF = XM_OFF + NG * 4 * KP_ROWS * 4;    // [groups][128 rows] (m, l)
    static constexpr int BAR_OFF = ML_OFF + NG * KP_ROWS * 8;
    static constexpr int BYTES = BAR_OFF + 8 * (3 * NB + NG + 2 + 4 * NS + 2);
    // The query rows' way to a row per thread: 4 KB a warp in the last QS value slots, which are filled after it.
    static constexpr int TURN = KVBYTES / 4096, QS = DP == 256 ? 1 : 2;
    static_assert(QS < NS && TURN * QS >= (DP == 64 ? 4 : 8), "the query rows fit those slots");
    static_assert(BYTES <= 227 * 1024, "fits an SM");
    static constexpr uint32_t TMEM_O = NB * KP_KEYS, TMEM_Q = TMEM_O + NG * DP, TMEM_COLS = 512;
    static_assert(TMEM_Q + DP / 2 <= TMEM_COLS, "scores, outputs and queries fit");
};

// OWN: some tiles take own rows (the kernel without them needs fewer registers: prefixes of 30016 keys of 8 KV heads took 43 us
// with it and 39 without).
template <int DP, bool OWN>
__global__ void __maxnreg__(KpSmem<DP>::REGS) k_kv_tiles_t5(const __grid_constant__ TileMaps maps,
                                                               const __grid_constant__ TileArgs a) {
    using L = KpSmem<DP>;
    constexpr int NS = L::NS, NG = L::NG, NB = L::NB, NDB = DP / 64;
    constexpr uint32_t IDESC_S = ptx::idesc_bf16_f32(KP_ROWS, KP_KEYS);
    constexpr uint32_t IDESC_PV = ptx::idesc_bf16_f32(KP_ROWS, DP) | (1u << 16);   // B MN-major
    extern __shared__ __align__(1024) uint8_t kp_smem[];
    uint8_t* stages = kp_smem;
    float* xmax = (float*)(kp_smem + L::XM_OFF);
    float2* ml = (float2*)(kp_smem + L::ML_OFF);
    uint64_t* bars = (uint64_t*)(kp_smem + L::BAR_OFF);
    uint64_t* sfull = bars;            // NB: score buffer ready
    uint64_t* pfull = sfull + NB;      // NB: probabilities written over the score buffer
    uint64_t* odone = pfull + NB;      // NB: P V of the block in score buffer b done
    uint64_t* gdone = odone + NB;      // NG: P V of the group's block done, of a block that another one of the group follows
    uint64_t* alldone = gdone + NG;    // every P V done
    uint64_t* qready = alldone + 1;    // the query rows are in TMEM
    uint64_t* kfull = qready + 1;      // NS each
    uint64_t* vfull = kfull + NS;
    uint64_t* kempty = vfull + NS;
    uint64_t* vempty = kempty + NS;
    uint32_t* tmem_slot = (uint32_t*)(vempty + NS);
    int* flag = (int*)(tmem_slot + 1);
    int* begun = flag + 1;             // NG: the group's output holds something before its first product

    const int tid = threadIdx.x, warp = ptx::warp_index(), lane = tid & 31;
    ptx::grid_dep_launch();
    const bool own = OWN && blockIdx.x >= a.side[0].blocks;
    const TileSide& sd = a.side[own];
    // Row tiles fastest: the blocks that read the same keys run together.
    uint32_t tile, split, kvh;
    const int cache = (int)a.c.by_K.div(sd.by_splits.div(sd.by_tiles.div(blockIdx.x - (own ? a.side[0].blocks : 0), tile), split), kvh);
    RowTile t;
    const int toks = own ? a.c.tokens : a.c.batch / a.c.groups * a.c.tokens;
    t.tok0 = (long long)cache * toks;
    t.head0 = (int)kvh * a.c.gq;
    t.R = toks * a.c.gq;
    t.r0 = (int)tile * KP_ROWS;
    // The tile's keys: rows of the run's prefix, then of the request's cache. Of the latter, `own_len` that some query row
    // of the tile sees and `own_low` that every one does.
    const int run = own ? (int)a.by_run.div((uint32_t)cache) : cache;
    const int pre_len = own && !a.both ? 0 : min(max(a.c.prefix.len[run], 0), a.c.prefix.rows);
    int own_len = 0, own_low = 0;
    if (own) {
        const int last = (int)a.c.by_gq.div((uint32_t)min(t.r0 + KP_ROWS, t.R) - 1);
        own_low = a.c.own.rows;
        for (int k = (int)a.c.by_gq.div((uint32_t)t.r0) + lane; k <= last; k += 32) {
            const int n = min(max(a.c.own.len[t.tok0 + k], 0), a.c.own.rows);
            own_len = max(own_len, n);
            own_low = min(own_low, n);
        }
        own_len = __reduce_max_sync(0xffffffffu, own_len);
        own_low = __reduce_min_sync(0xffffffffu, own_low);
    }
    // This block's key blocks, of the prefix's npre and then the own ones; none where they are fewer than the splits: the
    // part then weighs nothing.
    const int npre = (pre_len + KP_KEYS - 1) / KP_KEYS, nb_all = npre + (own_len + KP_KEYS - 1) / KP_KEYS;
    const int blk0 = (int)((long long)split * nb_all / sd.splits);
    const int nb = (int)((long long)(split + 1) * nb_all / sd.splits) - blk0;
    // Key (value) block i into its ring slot.
    auto load = [&](bool is_v, int i) {
        const int sl = i % NS, mine = OWN && blk0 + i >= npre, key0 = (blk0 + i - (mine ? npre : 0)) * KP_KEYS;
        uint64_t* full = (is_v ? vfull : kfull) + sl;
        uint8_t* base = stages + sl * L::STAGE + (is_v ? L::KVBYTES : 0);
        ptx::mbar_expect_tx(full, (uint32_t)L::KVBYTES);
        for (int db = 0; db < NDB; ++db)
            kv_load_box(base + db * (KP_KEYS * 128), is_v ? &maps.v[mine] : &maps.k[mine], full, db * 64, a.at[mine], (int)kvh, key0,
                        mine ? cache : run);
    };
    if (warp == 0 && ptx::elect_one()) {
        ptx::prefetch_tmap(&maps.k[OWN && blk0 >= npre]);
        ptx::prefetch_tmap(&maps.v[OWN && blk0 >= npre]);
        for (int b = 0; b < NB; ++b) {
            ptx::mbar_init(&sfull[b], 1);
            ptx::mbar_init(&pfull[b], KP_SOFT);
            ptx::mbar_init(&odone[b], 1);
        }
        for (int b = 0; b < NG; ++b) ptx::mbar_init(&gdone[b], 1);
        ptx::mbar_init(alldone, 1);
        ptx::mbar_init(qready, 256);
        for (int s = 0; s < NS; ++s) {
            ptx::mbar_init(&kfull[s], 1);
            ptx::mbar_init(&vfull[s], 1);
            ptx::mbar_init(&kempty[s], 1);
            ptx::mbar_init(&vempty[s], 1);
        }
        ptx::fence_mbar_init();
        *flag = 0;
        for (int b = 0; b < NG; ++b) begun[b] = 0;
        // The first use of the ring needs nothing of the other warps.
        for (int i = 0; i < NS && i < nb; ++i) {
            load(false, i);
            if (i < NS - L::QS) load(true, i);
        }
    }
    if (warp == 1) {
        ptx::tmem_alloc(tmem_slot, L::TMEM_COLS);
        ptx::tmem_relinquish();
    }
    // The softmax warps' query rows, on their way while the block sets itself up: 64-element blocks (warp - 4) / 4,
    // + 2, of the rows of the warp's TMEM lanes.
    constexpr int QN = (NDB + 1) / 2;
    uint4 qv[QN][8];
    if (warp >= 4 && warp < 12) {
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.c.q);
        // Row 4 i + (lane / 8): its token and head, stepped by 4 rows.
        int r = t.r0 + (warp & 3) * 32 + (lane >> 3);
        int tok = r / a.c.gq, hd = r - tok * a.c.gq;
        const int tok4 = 4 / a.c.gq, hd4 = 4 - tok4 * a.c.gq;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool in = r < t.R;
            const __nv_bfloat16* row = q + (in ? (t.tok0 + tok) * a.c.q_stride + (long long)(t.head0 + hd) * a.c.D : 0);
#pragma unroll
            for (int k = 0; k < QN; ++k) {
                const int d = 64 * (((warp - 4) >> 2) + 2 * k) + 8 * (lane & 7);
                qv[k][i] = kr_ld(row + d, in && d < a.c.D);
            }
            r += 4;
            tok += tok4;
            hd += hd4;
            if (hd >= a.c.gq) {
                hd -= a.c.gq;
                ++tok;
            }
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp <= 1) {
        if (ptx::elect_one()) {
            const bool is_v = warp == 1;
            uint64_t* fullb = is_v ? vfull : kfull;
            uint64_t* emptyb = is_v ? vempty : kempty;
            int issued = min(NS, nb);
            bool good = true;
            if (is_v) {
                good = ptx::mbar_wait_bounded(qready, 0, KP_WAIT_NS);
                if (!good) *flag = DEV_TIMEOUT_MMA;
                if (!good) issued = min(NS - L::QS, nb);
                for (int i = NS - L::QS; good && i < NS && i < nb; ++i) load(true, i);
            }
            for (int i = NS; good && i < nb; ++i) {
                if (!ptx::mbar_wait_bounded(&emptyb[i % NS], (i / NS - 1) & 1, KP_WAIT_NS)) {
                    *flag = DEV_TIMEOUT_WEIGHTS;
                    break;
                }
                load(is_v, i);
                issued = i + 1;
            }
            if (!ptx::ring_drain(fullb, NS, issued, KP_WAIT_NS)) *flag = DEV_TIMEOUT_WEIGHTS;
        }
    } else if (warp == 2) {
        if (ptx::elect_one()) {
            const uint32_t sb = ptx::smem_u32(stages);
            bool good = ptx::mbar_wait_bounded(qready, 0, KP_WAIT_NS);
            for (int i = 0; i < nb; ++i) {
                const int sl = i % NS;
                // (its score buffer holds P_{i-NB} until that product is done)
                if (i >= NB && good) good = ptx::mbar_wait_bounded(&odone[i % NB], (i / NB - 1) & 1, KP_WAIT_NS);
                if (good) good = ptx::mbar_wait_bounded(&kfull[sl], (i / NS) & 1, KP_WAIT_NS);
                ptx::tc_fence_after();
                if (good) {
                    const uint64_t kb = ptx::desc_sw128(sb + sl * L::STAGE);
#pragma unroll
                    for (int db = 0; db < NDB; ++db)
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            ptx::mma_bf16_ta(tmem + (uint32_t)(KP_KEYS * (i % NB)), tmem + L::TMEM_Q + (uint32_t)(8 * (4 * db + kk)),
                                             ptx::desc_add(kb, db * (KP_KEYS * 128) + kk * 32), IDESC_S, (db | kk) != 0);
                }
                ptx::mma_commit(&sfull[i % NB]);
                if (i + NS < nb) ptx::mma_commit(&kempty[sl]);
            }
            if (!good) *flag = DEV_TIMEOUT_MMA;
        }
    } else if (warp == 3) {
        if (ptx::elect_one()) {
            const uint32_t sb = ptx::smem_u32(stages);
            bool good = true;
            for (int i = 0; i < nb; ++i) {
                const int sl = i % NS;
                if (good) good = ptx::mbar_wait_bounded(&pfull[i % NB], (i / NB) & 1, KP_WAIT_NS);
                if (good) good = ptx::mbar_wait_bounded(&vfull[sl], (i / NS) & 1, KP_WAIT_NS);
                ptx::tc_fence_after();
                if (good) {
                    const uint64_t vb = ptx::desc_sw128_mn(sb + sl * L::STAGE + L::KVBYTES, KP_KEYS * 128, 1024);
#pragma unroll
                    for (int kk = 0; kk < KP_KEYS / 16; ++kk)
                        ptx::mma_bf16_ta(tmem + L::TMEM_O + (uint32_t)(i % NG * DP), tmem + (uint32_t)(KP_KEYS * (i % NB) + 8 * kk),
                                         ptx::desc_add(vb, kk * 16 * 128), IDESC_PV, i >= NG || kk != 0 || (OWN && begun[i] != 0));
                }
                if (i + NS < nb) ptx::mma_commit(&vempty[sl]);
                if (i + NB < nb) ptx::mma_commit(&odone[i % NB]);
                if (i + NG < nb) ptx::mma_commit(&gdone[i % NG]);
            }
            ptx::mma_commit(alldone);
            if (!good) *flag = DEV_TIMEOUT_MMA;
        }
    } else {
        const int grp = (warp - 4) >> 3, row = (warp & 3) * 32 + lane, half = ((warp - 4) >> 2) & 1;
        const int r = t.r0 + row;
        const bool valid = r < t.R;
        const int pre_vis = valid ? pre_len : 0;
        const int own_vis = valid && own ? min(max(a.c.own.len[row_token(a.c, t, r)], 0), a.c.own.rows) : 0;
        const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t out = lane_base + L::TMEM_O + (uint32_t)(grp * DP);
        const uint32_t pair_bar = 1 + 4 * grp + (warp & 3);   // the two warps of these 32 rows
        float m_used = -INFINITY, l = 0.f;          // m_used is the same in both threads of a row
        bool good = true;
        // The query rows were loaded 128 bytes of four rows an instruction: through 4 KB of shared memory of the warp
        // to a row per thread, then to TMEM (column 32 db + 4 c + e holds elements 64 db + 8 c + 2 e, + 1).
        if (grp == 0) {
            const int wi = warp - 4;
            uint4* turn = (uint4*)(stages + (NS - 1 - wi / L::TURN) * L::STAGE + L::KVBYTES + wi % L::TURN * 4096);
#pragma unroll
            for (int k = 0; k < QN; ++k) {
                const int db = half + 2 * k;
                if (db < NDB) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) turn[(4 * i + (lane >> 3)) * 8 + ((lane & 7) ^ ((4 * i + (lane >> 3)) & 7))] = qv[k][i];
                    __syncwarp();
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        uint32_t rq[16];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint4 v = turn[lane * 8 + ((4 * hf + c) ^ (lane & 7))];
                            rq[4 * c] = v.x;
                            rq[4 * c + 1] = v.y;
                            rq[4 * c + 2] = v.z;
                            rq[4 * c + 3] = v.w;
                        }
                        ptx::tmem_st_x16(lane_base + L::TMEM_Q + (uint32_t)(32 * db + 16 * hf), rq);
                    }
                    __syncwarp();
                }
            }
            ptx::tmem_st_wait();
            ptx::fence_proxy_async_smem();   // the slots' values land after these accesses
            ptx::tc_fence_before();
            ptx::mbar_arrive(qready);
        }
        constexpr int HK = KP_KEYS / 2;   // keys per thread
        const uint64_t c2 = pair2(a.c2);
        const float rescale = KP_RESCALE / a.c2;
        for (int i = grp; i < nb; i += NG) {
            if (good) good = ptx::mbar_wait_bounded(&sfull[i % NB], (i / NB) & 1, KP_WAIT_NS);
            ptx::tc_fence_after();
            uint32_t s[2][16];
            {
                const uint32_t sa = lane_base + (uint32_t)(KP_KEYS * (i % NB) + HK * half);
                ptx::tmem_ld_x16(sa, s[0]);
                ptx::tmem_ld_x16(sa + 16u, s[1]);
                ptx::tmem_ld_wait();
            }
            // Keys of the block: its first one, and of this half the ones that the row sees.
            const bool theirs = OWN && blk0 + i >= npre;   // own rows
            const int key0 = (blk0 + i - (theirs ? npre : 0)) * KP_KEYS;
            const int vis = (theirs ? own_vis : pre_vis) - key0 - HK * half;
            const bool full = __all_sync(0xffffffffu, vis >= HK);
            if (!full) {
#pragma unroll
                for (int j = 0; j < HK; ++j)
                    if (j >= vis) s[j >> 4][j & 15] = __float_as_uint(-INFINITY);
            }
            float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int j = 0; j < HK; ++j) m4[j & 3] = fmaxf(m4[j & 3], __uint_as_float(s[j >> 4][j & 15]));
            float mb = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            float* xm = xmax + (2 * grp + (i / NG & 1)) * 2 * KP_ROWS + row;
            xm[half * KP_ROWS] = mb;
            ptx::named_bar_sync(pair_bar, 64);
            mb = fmaxf(mb, xm[(1 - half) * KP_ROWS]);
            const bool move = mb > m_used + rescale;
            const float alpha = !move ? 1.f : m_used == -INFINITY ? 0.f : kr_ex2((m_used - mb) * a.c2);
            // TMEM accesses are warp-collective: the warp rescales together (its half of the columns), lanes whose
            // maximum stays put multiply by 1. O is settled once P V of the group's previous block is done.
            if (__any_sync(0xffffffffu, move && i >= NG && m_used != -INFINITY)) {
                if (good) good = ptx::mbar_wait_bounded(&gdone[grp], (i / NG - 1) & 1, KP_WAIT_NS);
                ptx::tc_fence_after();
#pragma unroll 1
                for (int c0 = half * (DP / 2); c0 < (half + 1) * (DP / 2); c0 += 16) {
                    uint32_t ro[16];
                    ptx::tmem_ld_x16(out + (uint32_t)c0, ro);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) ro[j] = __float_as_uint(__uint_as_float(ro[j]) * alpha);
                    ptx::tmem_st_x16(out + (uint32_t)c0, ro);
                }
                ptx::tmem_st_wait();
            }
            if (move) {
                l *= alpha;
                m_used = mb;
            }
            // 2^((s - m) c): a hidden key's -inf gives 0, also while the row has seen none at all (m taken as 0).
            const uint64_t neg_m = pair2(m_used == -INFINITY ? 0.f : -m_used);
            float l4[4] = {0.f, 0.f, 0.f, 0.f};
            uint32_t pk[HK / 2];
#pragma unroll
            for (int k = 0; k < HK; k += 2) {
                float p0, p1;
                sub_scale2(__uint_as_float(s[k >> 4][k & 15]), __uint_as_float(s[k >> 4][(k + 1) & 15]), neg_m, c2, p0, p1);
                p0 = kr_ex2(p0);
                p1 = kr_ex2(p1);
                l4[(k >> 1) & 3] += p0 + p1;
                pk[k / 2] = kr_pack(p0, p1);
            }
            l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
            const int live = (theirs ? own_len : pre_len) - key0;   // keys of the block that some row sees; the same for all threads
            if (OWN && theirs && own_low < min(own_len, key0 + KP_KEYS)) {
                // Some rows see a part of them only: is there an infinity or NaN among the values?
                const int sl = i % NS;
                if (good) good = ptx::mbar_wait_bounded(&vfull[sl], (i / NS) & 1, KP_WAIT_NS);
                uint8_t* vb = stages + sl * L::STAGE + L::KVBYTES;
                bool odd = false;
                for (int e = (tid - 128) % KP_SOFT; e < min(live, KP_KEYS) * NDB * 8; e += KP_SOFT) {
                    const int key = e / (NDB * 8), p = e % (NDB * 8);
                    const uint4 v = *(const uint4*)(vb + (p / 8) * (KP_KEYS * 128) + key * 128 + (p % 8) * 16);
                    odd = odd || bad_pair(v.x) || bad_pair(v.y) || bad_pair(v.z) || bad_pair(v.w);
                }
                if (group_any(11 + grp, KP_SOFT, odd)) {
                    // Row by row: first one half's keys, then the other's, onto the settled output of the blocks before.
                    if (i >= NG && good) good = ptx::mbar_wait_bounded(&gdone[grp], (i / NG - 1) & 1, KP_WAIT_NS);
                    ptx::tc_fence_after();
                    for (int turn = 0; turn < 2; ++turn) {
                        if (turn == half) {
#pragma unroll 1
                            for (int c0 = 0; c0 < DP; c0 += 16) {
                                uint32_t ro[16];
                                if (i < NG && turn == 0) {
#pragma unroll
                                    for (int j = 0; j < 16; ++j) ro[j] = 0u;
                                } else {
                                    ptx::tmem_ld_x16(out + (uint32_t)c0, ro);
                                    ptx::tmem_ld_wait();
                                }
#pragma unroll
                                for (int k = 0; k < HK; ++k) {
                                    if (k >= vis) continue;
                                    const int key = HK * half + k;
                                    const float pr = __uint_as_float(k & 1 ? pk[k / 2] & 0xffff0000u : pk[k / 2] << 16);
                                    const uint8_t* vr = vb + (c0 / 64) * (KP_KEYS * 128) + key * 128;
#pragma unroll
                                    for (int h = 0; h < 2; ++h) {
                                        const uint4 v = *(const uint4*)(vr + (((c0 % 64 / 8 + h) ^ (key & 7)) << 4));
                                        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                        for (int e = 0; e < 4; ++e) {
                                            uint32_t &y0 = ro[8 * h + 2 * e], &y1 = ro[8 * h + 2 * e + 1];
                                            y0 = __float_as_uint(fmaf(pr, __uint_as_float(x[e] << 16), __uint_as_float(y0)));
                                            y1 = __float_as_uint(fmaf(pr, __uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y1)));
                                        }
                                    }
                                }
                                __syncwarp();
                                ptx::tmem_st_x16(out + (uint32_t)c0, ro);
                            }
                            ptx::tmem_st_wait();
                            ptx::tc_fence_before();
                        }
                        ptx::named_bar_sync(pair_bar, 64);
                        ptx::tc_fence_after();
                    }
#pragma unroll
                    for (int k = 0; k < HK / 2; ++k) pk[k] = 0u;
                    ptx::named_bar_sync(11 + grp, KP_SOFT);   // every thread has read the values
                    for (int e = (tid - 128) % KP_SOFT; good && e < KP_KEYS * NDB * 8; e += KP_SOFT) ((uint4*)vb)[e] = make_uint4(0, 0, 0, 0);
                    if (i < NG && tid % KP_SOFT == 128) begun[grp] = 1;
                    ptx::fence_proxy_async_smem();
                }
            }
            // Over the scores of both halves: both threads of a row have read theirs (the barrier above). Column 16 half
            // + e holds keys 32 half + 2 e, + 1.
            ptx::tmem_st_x16(lane_base + (uint32_t)(KP_KEYS * (i % NB) + 16 * half), pk);
            ptx::tmem_st_wait();
            if (live < KP_KEYS) {
                // Values of rows past the end, as they landed: cleared (a row's 16-byte pieces stay in the row).
                const int sl = i % NS;
                if (good) good = ptx::mbar_wait_bounded(&vfull[sl], (i / NS) & 1, KP_WAIT_NS);
                uint8_t* vb = stages + sl * L::STAGE + L::KVBYTES;
                for (int e = (tid - 128) % KP_SOFT; good && e < (KP_KEYS - live) * NDB * 8; e += KP_SOFT) {
                    const int key = live + e / (NDB * 8), p = e % (NDB * 8);
                    *(uint4*)(vb + (p / 8) * (KP_KEYS * 128) + key * 128 + (p % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                ptx::fence_proxy_async_smem();
            }
            ptx::tc_fence_before();
            ptx::mbar_arrive(&pfull[i % NB]);
        }
        // The row's sum: both halves, in order, through the buffer that the last block's maxima are not in.
        const int mine = (nb - grp + NG - 1) / NG;   // blocks of this group
        float* xl = xmax + (2 * grp + (mine & 1)) * 2 * KP_ROWS + row;
        xl[half * KP_ROWS] = l;
        ptx::named_bar_sync(pair_bar, 64);
        l = xl[0] + xl[KP_ROWS];
        // Every P V of the block is done, and with them every read of the ring. (The groups' own barriers cannot tell: the
        // last scores came when up to two products of a group were still to run.)
        if (good) good = ptx::mbar_wait_bounded(alldone, 0, KP_WAIT_NS);
        ptx::tc_fence_after();
        if (!good) *flag = DEV_TIMEOUT_MMA;
        // The groups' outputs are joined on the way: w_g = 2^((m_g - M) c).
        float w = 1.f;
        if (NG > 1) {
            if (half == 0) ml[grp * KP_ROWS + row] = make_float2(m_used, l);
            ptx::named_bar_sync(9, NG * KP_SOFT);
            const float2 other = ml[(1 - grp) * KP_ROWS + row];
            const float M = fmaxf(m_used, other.x);
            w = m_used == -INFINITY ? 0.f : kr_ex2((m_used - M) * a.c2);
            l = w * l + (other.x == -INFINITY ? 0.f : kr_ex2((other.x - M) * a.c2)) * other.y;   // (0 times a NaN sum is NaN)
            m_used = M;
        }
        // A result is scaled by 1 / l and rounded on its way; a half row's 16-bit values go where its own 32-bit ones were.
        const float inv = l == 0.f ? 0.f : 1.f / l;   // (0: the row saw no key; a NaN score makes l, and so the row, NaN)
        uint8_t* orow = kp_smem + row * L::OUT_LD;
#pragma unroll 1
        for (int turn = 0; turn < NG; ++turn) {
            if (turn == grp) {
#pragma unroll 1
                for (int c0 = half * (DP / 2); c0 < (half + 1) * (DP / 2); c0 += 32) {
                    uint32_t v[2][16];
                    ptx::tmem_ld_x16(out + (uint32_t)c0, v[0]);
                    ptx::tmem_ld_x16(out + (uint32_t)(c0 + 16), v[1]);
                    ptx::tmem_ld_wait();
                    // (a wait that gave up may have left copies on their way into the ring)
                    if (good && (mine > 0 || (a.out && nb > 0))) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            uint4* dst = (uint4*)(orow + (c0 + 4 * k) * 4);
                            float x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                x[e] = __uint_as_float(v[k >> 2][4 * (k & 3) + e]);
                                if (NG > 1) x[e] = mine > 0 ? w * x[e] : 0.f;
                            }
                            if (grp > 0) {
                                const uint4 y = *dst;
                                x[0] += __uint_as_float(y.x);
                                x[1] += __uint_as_float(y.y);
                                x[2] += __uint_as_float(y.z);
                                x[3] += __uint_as_float(y.w);
                            }
                            if (a.out && grp == NG - 1) {
                                uint32_t* dst16 = (uint32_t*)(orow + half * (DP * 2) + (c0 + 4 * k - half * (DP / 2)) * 2);
                                dst16[0] = kr_pack(x[0] * inv, x[1] * inv);
                                dst16[1] = kr_pack(x[2] * inv, x[3] * inv);
                            } else {
                                *dst = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
                            }
                        }
                    }
                }
            }
            if (turn + 1 < NG) ptx::named_bar_sync(10, NG * KP_SOFT);
        }
        if (grp < NG - 1) {
            ptx::grid_dep_wait();
        } else {
            ptx::fence_proxy_async_smem();
            ptx::named_bar_sync(pair_bar, 64);
            ptx::grid_dep_wait();   // the row kernel that started before this one: what waits for this kernel has both
            if (half == 0 && valid) {
                const long long row_at = row_index(a.c, t, r), row_out = (sd.part0 + (long long)split) * a.rows + row_at;
                auto copy = [&](void* dst, const uint8_t* src, int bytes) {
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(ptx::smem_u32(src)),
                                 "r"(bytes)
                                 : "memory");
                };
                if (a.out) {
                    __nv_bfloat16* dst = a.out + row_at * a.c.D;
                    if (a.lse) a.lse[row_at] = l == 0.f ? -INFINITY : fmaf(m_used, a.c.scale, logf(l));
                    if (nb == 0) {
                        for (int d = 0; d < a.c.D; d += 8) *(uint4*)(dst + d) = make_uint4(0, 0, 0, 0);
                    } else if (good) {
                        copy(dst, orow, min(a.c.D, DP / 2) * 2);
                        if (a.c.D > DP / 2) copy(dst + DP / 2, orow + DP * 2, (a.c.D - DP / 2) * 2);
                    }
                } else {
                    a.pml[row_at * a.parts + sd.part0 + split] = make_float2(m_used, l);
                    if (good && nb > 0) copy(a.po + row_out * a.c.D, orow, a.c.D * 4);
                }
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            }
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (tid == 0 && *flag != 0) atomicCAS(a.err, 0, *flag);
    if (warp == 1) ptx::tmem_dealloc(tmem, L::TMEM_COLS);
}

template <int DP>
jpi_status launch_dim(const TileArgs& a, const TileMaps& m, bool early, cudaStream_t st) {
    return kv_start(a.side[1].blocks > 0 ? k_kv_tiles_t5<DP, true> : k_kv_tiles_t5<DP, false>,
                    dim3(a.side[0].blocks + a.side[1].blocks), KpSmem<DP>::THREADS, KpSmem<DP>::BYTES, early, st, m, a);
}

template <int DP>
jpi_status prepare_dim() {
    for (auto* kernel : {k_kv_tiles_t5<DP, false>, k_kv_tiles_t5<DP, true>}) {
        JPI_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, KpSmem<DP>::BYTES));
        // An SM that runs a block of the row kernel takes one of these beside it only if both want it set up alike.
        JPI_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    }
    return JPI_OK;
}

// What the tiles would make of a side: row tiles over all runs or requests and KV heads, and key blocks of each.
struct TileWork {
    bool fit = false;
    long long tiles = 0, blocks = 0, nb = 0;
    long long elements = 0;   // of keys that the row kernel would read: each row of 8 query rows' tile by itself
};
TileWork work_of(const jpi_kv_handle* h, const KvCall& c, bool own) {
    TileWork w;
    const KvSide& s = own ? c.own : c.prefix;
    if (!h->bf16 || c.D < 64 || s.rows == 0) return w;
    const int caches = own ? c.batch : c.groups;
    const long long R = (long long)(own ? 1 : c.batch / c.groups) * c.tokens * c.gq;
    KvMapDims m;
    if (h->tiles == 0 || (h->tiles < 0 && R < kp_least(own, c.D)) || !kv_map_dims(s, c.K, c.D, caches, &m)) return w;
    w.tiles = (R + KP_ROWS - 1) / KP_ROWS;
    w.blocks = w.tiles * c.K * caches;
    w.nb = (s.rows + KP_KEYS - 1) / KP_KEYS;
    w.fit = w.blocks * w.nb < (1ll << 31);
    w.elements = (R + 7) / 8 * c.K * caches * s.rows * c.D;
    return w;
}

// Key blocks' time that s splits of each of `blocks` tiles take with `rest` of other work to share the SMs with.
long long tiles_time(const jpi_kv_handle* h, const TileWork& w, long long s, long long rest) {
    const long long u = (w.nb + s - 1) / s + KP_FIXED;
    return std::max((w.blocks * s + h->num_sms - 1) / h->num_sms * u, (w.blocks * s * u + rest) / h->num_sms);
}
// What a result in `parts` parts costs beside one written by its tiles, in the same unit: rows of 32 bits to the
// workspace, the combine's launch, and the rows read back (about 4 MB in a key block's time). One part and two of the 16
// chunks of 51 tokens over prefixes of 816 keys: 23 and 26 us.
long long join_time(const KvCall& c, long long parts) {
    return 7 + parts * ((long long)c.batch * c.tokens * c.H * c.D * 4 >> 10) / 3900;
}

}  // namespace

jpi_status kv_tiles_prepare(jpi_kv_handle* h) {
    if (!h->bf16 || h->D < 64) return JPI_OK;
    return h->D <= 64 ? prepare_dim<64>() : h->D <= 128 ? prepare_dim<128>() : prepare_dim<256>();
}

void kv_tiles_plan(const jpi_kv_handle* h, const KvCall& c, long long room, KvTilesPlan* plan) {
    TileWork p = work_of(h, c, false), o = work_of(h, c, true);
    *plan = KvTilesPlan();
    if (h->tiles < 0 && (p.fit ? p.elements : 0) + (o.fit ? o.elements : 0) <= KP_ROW_ELEMENTS) return;
    auto splits_most = [&](const TileWork& w) { return std::min({w.nb, room, std::max(1ll, 2ll * h->num_sms / w.blocks)}); };
    // The side of more work is split so that its blocks, or the waves of them, end first; the other to blocks no longer.
    const bool own_first = o.fit && (!p.fit || o.blocks * o.nb > p.blocks * p.nb);
    const TileWork &a = own_first ? o : p, &b = own_first ? p : o;
    if (!a.fit) return;
    long long best = 1, best_time = -1, best_b = 0;
    for (long long s = 1; s <= splits_most(a); ++s) {
        const long long u = (a.nb + s - 1) / s;
        const long long sb = b.fit ? std::min(room, (b.nb + u - 1) / u) : 0;
        const long long rest = b.fit ? b.blocks * sb * ((b.nb + sb - 1) / sb + KP_FIXED) : 0;
        const bool more = c.prefix.rows > 0 && c.own.rows > 0;   // parts of the other side, tiles or not
        const long long time = tiles_time(h, a, s, rest) + (s + sb + more > 1 ? join_time(c, s + std::max<long long>(sb, more)) : 0);
        if (best_time < 0 || time < best_time) {
            best = s;
            best_time = time;
            best_b = sb;
        }
    }
    plan->splits[own_first] = (int)best;
    plan->splits[!own_first] = (int)best_b;
    // Both sides by the requests' tiles, where that is estimated to end earlier: no tile is shared between requests, but
    // a single split needs no combine.
    if (p.fit && o.fit) {
        TileWork w = o;
        w.nb += p.nb;
        for (long long s = 1; s <= splits_most(w); ++s) {
            const long long time = tiles_time(h, w, s, 0) + (s > 1 ? join_time(c, s) : 0);
            if (time <= best_time) {
                best_time = time;
                plan->both = true;
                plan->splits[0] = 0;
                plan->splits[1] = (int)s;
            }
        }
    }
}

jpi_status launch_kv_tiles_t5(jpi_kv_handle* h, const KvCall& c, const KvTilesPlan& plan, const int part0[2], float* po,
                              float2* pml, int parts, void* out, float* lse, bool early, cudaStream_t st) {
    TileArgs a = {};
    TileMaps maps = {};
    a.c = c;
    a.c2 = KR_LOG2E * c.scale;
    a.both = plan.both;
    a.by_run = KvDiv((uint32_t)(c.batch / c.groups));
    a.po = po;
    a.pml = pml;
    a.parts = parts;
    a.rows = (long long)c.batch * c.tokens * c.H;
    a.out = parts == 1 ? static_cast<__nv_bfloat16*>(out) : nullptr;
    a.lse = lse;
    a.err = h->dev_err;
    for (int i = 0; i < 2; ++i) {
        if (plan.splits[i] > 0) {
            const TileWork w = work_of(h, c, i == 1);
            TileSide& d = a.side[i];
            d.splits = plan.splits[i];
            d.tiles = (int)w.tiles;
            d.part0 = part0[i];
            d.blocks = (uint32_t)(w.blocks * d.splits);
            d.by_splits = KvDiv((uint32_t)d.splits);
            d.by_tiles = KvDiv((uint32_t)d.tiles);
        } else if (!(i == 0 && plan.both)) {
            continue;
        }
        const KvSide& s = i ? c.own : c.prefix;
        KvMapDims m;
        if (!kv_map_dims(s, c.K, c.D, i ? c.batch : c.groups, &m) || !kv_make_map(m, s.k, c.D, KP_KEYS, &maps.k[i]) ||
            !kv_make_map(m, s.v, c.D, KP_KEYS, &maps.v[i])) {
            set_error("cuTensorMapEncodeTiled refused the %s", i ? "own rows" : "prefix");
            return JPI_ERR_CUDA;
        }
        a.at[i] = make_int3(m.at_head, m.at_row, m.at_cache);
    }
    return c.D <= 64 ? launch_dim<64>(a, maps, early, st) : c.D <= 128 ? launch_dim<128>(a, maps, early, st) : launch_dim<256>(a, maps, early, st);
}

}  // namespace jpi
