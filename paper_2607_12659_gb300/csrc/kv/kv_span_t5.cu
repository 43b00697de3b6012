// Attention over windows with many query rows on tcgen05 (kv_span.h): 128 query rows (tokens x heads of one KV head of a
// request) per block over a range of the key blocks of 64 that its tokens see.
//   warp 0  bf16 caches, one thread: K blocks by bulk tensor copies into a ring of NS slots
//   warp 1  the same for V
//   warp 2  one thread: S_i = Q K_i^T (M = 128, N = 64, K = D) into one of NB TMEM score buffers
//   warp 3  one thread: O += P_i V_i (M = 128, N = D, K = 64), V read as an MN-major operand
//   warps 4-  groups of eight: two threads per query row, half of a block's keys each: maximum, 2^x, probabilities back to
//           tensor memory, over the scores they come from. To D = 128 two groups take the even and the odd blocks, each with a
//           maximum, sum and output of its own, joined at the end. At D = 256 tensor memory holds one output and two score buffers,
//           which a block keeps for twice the time of a softmax, so that a second group would wait. O is rescaled only when a block's maximum passes the running one by more
//           than ST_RESCALE.
//   8-bit caches: four more warps read codes ahead into registers and write them to the ring's slots as fp16 numbers, which
//           e4m3 is a subset of: one instruction for two, half a tile's shared-memory writes a thread. Then both products take fp16: the
//           queries at a power of two of each row's own (that its maximum and scale know of), the probabilities times
//           the scale of their block's values relative to the largest 2^e that the row has seen, p 2^(e_j - e) 2^4 <= 2^15. (As bf16
//           numbers with the scales in them the codes would take five instructions more a pair, which the softmax needs.)
// The query rows are gathered by the softmax threads into tensor memory as the A operand of the score products.
//
// Probabilities are rounded to the operands' type once: each off by at most 2^-8 of itself; in fp16 2^-11, or 2^-29 times 2^(e - e_j).
//
// Rows of the cache that no query row of the tile sees may hold anything: their scores are replaced, and their values are
// cleared in shared memory before the product, since 0 times a NaN would reach every row. Blocks that only some of the query
// rows see whole are searched for infinities and NaN; one that holds any is added row by row on CUDA cores instead (each row
// its own keys), and the product adds nothing. A row that sees nothing has l = 0, and what its outputs hold is not used.
//
// Each block leaves a part (unnormalised fp32 rows, (m, l)) for the combine, or the result: rows pass through shared
// memory (the ring, free by then). Of two parts whose pairs of blocks are all resident together (JOIN) the pair is a cluster, and each of
// its blocks joins and writes half of the rows from both shared memories: 16 x 51 tokens over 867 rows in 8 bits 31.6 us with the
// combine, 23.7 so; 256 tokens of 32 heads on 8 over 2100 keys 28.4 and 20.4.
//
// Every wait is bounded; a wait that gives up records an error in the handle's word, and its thread waits for
// nothing more.

#include "kv_tiles.cuh"
#include "kv8.cuh"
#include "kv_maps.h"
#include "kv_span.cuh"

#include <algorithm>

namespace jpi {
namespace {

constexpr int ST_ROWS = 128;
constexpr int ST_KEYS = 64;
constexpr int ST_SOFT = 256;    // threads of a softmax group
constexpr int ST_CONV = 128;    // threads that write codes to the ring: half of them keys, half values
constexpr uint64_t ST_WAIT_NS = 200ull * 1000 * 1000;
// How far a block's maximum passes the running one, in log2 units, before the outputs are rescaled, which takes longer than a block's
// softmax: a probability of bf16 has fp32's range, and the sums have room for 2^24 times what they would be. One of fp16 is at most
// 2^ST_RESCALE8 ST_BOOST.
constexpr float ST_RESCALE = 24.f, ST_RESCALE8 = 11.f;
constexpr int ST_BOOST = 4;         // log2 of what probabilities of fp16 are multiplied by
constexpr int ST_NONE = -4096;      // no scale seen yet
constexpr int ST_RUN = 32;          // blocks of a group whose scales are read together
constexpr int ST_RANKS = 2;         // parts that are joined in a cluster
// Query rows of a request and KV head from which a call that has no room in clusters (kv_span.cu) takes the tiles, and the elements of keys up
// to which it stays with the row kernel all the same, which reads a key once for every 8 query rows: what the row kernel takes grows with
// both, what a tile takes by its keys alone, however few of its rows there are and however narrow the heads. Microseconds of row kernel
// and tiles, 8 bits, 32 KV heads to D = 128 and 8 at 256:
//   D = 64   64 rows over 4096 keys (64 M elements) 27.3 and 29.0, over 16384 (256 M) 78 and 82, 32 rows 43 and 85; 96 rows over 1024
//            (24 M) 17.6 and 18.6, over 2048 24.2 and 22.4; 128 rows over 512 (16 M) 15.8 and 14.8
//   D = 128  32 rows over 2048 (32 M) 19.3 and 21.0, over 16384 81 and 88; 40 rows over 1024 (20 M) 15.7 and 16.7; 56 rows over 1024 (28 M)
//            18.7 and 17.0; 64 rows over 512 (16 M) 13.6 and 15.4, over 1024 20.0 and 16.9
//   D = 256  40 rows over 1024 (10 M) 13.5 and 14.4, over 2048 16.5 and 15.9; 64 rows of one KV head over 4096 (8 M) 12.4 and 14.3, over 16384
//            19.4 and 16.7
// and bf16:
//   D = 64   32 rows over 2048 (16 M) 12.8 and 15.0, over 16384 42 and 54; 48 rows over 1024 (12 M) 12.1 and 13.5, over 2048 15.7 and 15.4
//   D = 128  48 rows over 512 (12 M) 12.4 and 13.6, over 1024 15.8 and 14.8; 64 rows of 8 KV heads over 1024 (8 M) 10.6 and 11.8, over 4096
//            17.5 and 13.9
//   D = 256  128 rows of one KV head over 1024 (4 M) 10.9 and 12.1, 64 over 4096 (8 M) 12.1 and 11.9, over 16384 19.8 and 14.3
constexpr int ST_LEAST = 32;
constexpr long long ST_NEVER = 1ll << 62;
constexpr long long st_row_elements(bool held8, long long R, int D) {
    if (held8) return D > 128 ? 12ll << 20 : D > 64 ? (R < 36 ? ST_NEVER : (R < 64 ? 20ll : 16ll) << 20) : R < 72 ? ST_NEVER : (R < 128 ? 24ll : 12ll) << 20;
    return D > 128 ? 4ll << 20 : D <= 64 && R < 44 ? ST_NEVER : 12ll << 20;
}
// Cycles of a key block of D elements, of a block's start and end, of the combine's launch, of a pair's meeting, and bytes a cycle to and from
// the workspace.
constexpr long long st_block(bool held8, int D) { return held8 ? 1000 + 8 * D : 500 + 4 * D; }
constexpr long long ST_ENDS = 10000, ST_JOIN = 8000, ST_BYTES = 2600;
constexpr long long st_meet(int D) { return 3000 + 14 * D; }

struct SpanMaps {
    CUtensorMap k, v;
};
struct SpanTileArgs {
    KvCall c;
    KvSpan s;
    float c2;              // log2(e) * scale
    int splits, tiles;     // key ranges, row tiles of a request and KV head
    KvDiv by_splits, by_tiles, by_rest;   // (rest: splits of all caches and KV heads)
    bool tiles_outer;
    int3 at;               // of the maps' outer dimensions: heads, rows, caches
    float* po;             // [parts][rows][D]
    float2* pml;           // [rows][parts]
    long long rows;
    __nv_bfloat16* out;    // of a call of one part: the result, else null
    __nv_bfloat16* joined; // of one whose two parts are joined in clusters: the result, else null
    float* lse;
    int* err;
};

template <int DP, bool Q8>
struct StSmem {
    static constexpr int NS = Q8 ? (DP == 256 ? 2 : 3) : DP == 256 ? 3 : 5;
    static constexpr int KVBYTES = ST_KEYS * DP * 2;
    static constexpr int STAGE = 2 * KVBYTES;               // ring slot: K, then V
    static constexpr int OUT_LD = DP * 4 + 16;              // bytes of a staged output row: the pad spreads the banks
    static constexpr int RING = NS * STAGE > ST_ROWS * OUT_LD ? NS * STAGE : ST_ROWS * OUT_LD;
    static constexpr int NG = DP == 256 ? 1 : 2;            // softmax groups
    static constexpr int CONV = 128 + NG * ST_SOFT;         // first thread of those that convert
    static constexpr int THREADS = CONV + (Q8 ? ST_CONV : 0);
    static constexpr int REGS = 65536 / THREADS / 8 * 8;
    static constexpr int NB = DP == 256 ? 2 : 3;            // score buffers
    static constexpr int RAW = DP == 256 ? 2 : 4;           // 8 bits: blocks of codes on their way
    static constexpr int RAWBYTES = ST_KEYS * DP * 2;       // of a block's keys and values
    static constexpr int XM_OFF = RING + (Q8 ? RAW * RAWBYTES : 0);   // [groups][2 blocks][2 key halves][128 rows]
    static constexpr int ML_OFF = XM_OFF + NG * 4 * ST_ROWS * 4;    // [groups][128 rows] (m, l)
    static constexpr int QM_OFF = ML_OFF + NG * ST_ROWS * 8;        // [2 halves of d][128 rows] largest |q|
    static constexpr int SC_OFF = QM_OFF + 2 * ST_ROWS * 4;         // [groups][ST_RUN blocks] scales of a block's four tiles: keys, values
    static constexpr int BAR_OFF = SC_OFF + NG * ST_RUN * 8;
    static constexpr int BYTES = BAR_OFF + 8 * (3 * NB + NG + 2 + 4 * NS + 2);
    // The query rows' way to a row per thread: 4 KB a warp in the last QS value slots, which are filled after it.
    static constexpr int TURN = KVBYTES / 4096, QS = DP == 256 ? 1 : 2;
    static_assert(QS < NS && TURN * QS >= (DP == 64 ? 4 : 8), "the query rows fit those slots");
    static_assert(BYTES <= 227 * 1024 && THREADS * REGS <= 65536, "fits an SM");
    static constexpr uint32_t TMEM_O = NB * ST_KEYS, TMEM_Q = TMEM_O + NG * DP, TMEM_COLS = 512;
    static_assert(TMEM_Q + DP / 2 <= TMEM_COLS, "scores, outputs and queries fit");
};

__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Joins the parts of a tile, staged in the shared memories of the cluster's blocks, and writes the rows of block `rank`. What
// bounds it is the latency of reads from the other block, so that eight of 16 bytes a lane, of several rows, are on their way together.
template <int DP, int LD, int WARPS>
__device__ __forceinline__ void join_tile(const SpanTileArgs& a, const RowTile& t, int rank, const uint8_t* rows, const float2* ml, int warp, int lane) {
    constexpr int RANKS = ST_RANKS, CH = DP > 128 ? 2 : 1, RW = 8 / RANKS / CH;   // 128-element parts of a row; rows together
    constexpr int step = RANKS * WARPS;
    for (int r0 = rank + RANKS * warp; r0 < ST_ROWS; r0 += RW * step) {
        float2 part[RW][RANKS];
        float4 v[RW][CH][RANKS];
#pragma unroll
        for (int u = 0; u < RW; ++u)
#pragma unroll
            for (int k = 0; k < RANKS; ++k) {
                const int r = r0 + u * step;
                part[u][k] = make_float2(-INFINITY, 0.f);
                if (r >= ST_ROWS || t.r0 + r >= t.R) continue;
                part[u][k] = ptx::dsmem_ld_f2(ptx::dsmem_map(ptx::smem_u32(ml + r), (uint32_t)k));
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    v[u][c][k] = ptx::dsmem_ld_f4(ptx::dsmem_map(ptx::smem_u32(rows + r * LD + 16 * min(lane + 32 * c, DP / 4 - 1)), (uint32_t)k));
            }
#pragma unroll
        for (int u = 0; u < RW; ++u) {
            const int r = r0 + u * step;
            if (r >= ST_ROWS || t.r0 + r >= t.R) continue;
            const long long row_at = row_index(a.c, t, t.r0 + r);
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int k = 0; k < RANKS; ++k) m = fmaxf(m, part[u][k].x);
            float4 x[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) x[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < RANKS; ++k) {
                if (part[u][k].y == 0.f) continue;   // a part without a sum holds nothing
                const float w = part[u][k].x == -INFINITY ? 0.f : kr_ex2((part[u][k].x - m) * a.c2);
                l = fmaf(w, part[u][k].y, l);
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const float4 y = v[u][c][k];
                    x[c] = make_float4(fmaf(w, y.x, x[c].x), fmaf(w, y.y, x[c].y), fmaf(w, y.z, x[c].z), fmaf(w, y.w, x[c].w));
                }
            }
            const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int d = 4 * (lane + 32 * c);
                if (d < a.c.D)
                    *(uint2*)(a.joined + row_at * a.c.D + d) = make_uint2(kr_pack(x[c].x * inv, x[c].y * inv), kr_pack(x[c].z * inv, x[c].w * inv));
            }
            if (lane == 0 && a.lse) a.lse[row_at] = l == 0.f ? -INFINITY : fmaf(m, a.c.scale, logf(l));
        }
    }
}

template <int DP, bool Q8, bool JOIN>
__global__ void __maxnreg__((StSmem<DP, Q8>::REGS)) k_kv_span_t5(const __grid_constant__ SpanMaps maps,
                                                               const __grid_constant__ SpanTileArgs a) {
    using L = StSmem<DP, Q8>;
    constexpr int NS = L::NS, NG = L::NG, NB = L::NB, NDB = DP / 64;
    // (fp16 operands are type 0 of both fields)
    constexpr uint32_t TYPES = Q8 ? ~((1u << 7) | (1u << 10)) : ~0u;
    constexpr uint32_t IDESC_S = ptx::idesc_bf16_f32(ST_ROWS, ST_KEYS) & TYPES;
    constexpr uint32_t IDESC_PV = (ptx::idesc_bf16_f32(ST_ROWS, DP) | (1u << 16)) & TYPES;   // B MN-major
    extern __shared__ __align__(1024) uint8_t st_smem[];
    uint8_t* stages = st_smem;
    float* xmax = (float*)(st_smem + L::XM_OFF);
    float2* ml = (float2*)(st_smem + L::ML_OFF);
    float* qmax = (float*)(st_smem + L::QM_OFF);
    uint64_t* bars = (uint64_t*)(st_smem + L::BAR_OFF);
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
    // The last row tiles first, whose tokens see most: of all caches together where their keys stay in L2, else of one after the other, so
    // that the blocks that read the same keys run together.
    uint32_t tile, split, kvh, rest;
    if (a.tiles_outer) tile = a.by_rest.div(blockIdx.x, rest);
    else rest = a.by_tiles.div(blockIdx.x, tile);
    tile = (uint32_t)a.tiles - 1 - tile;
    const int cache = (int)a.c.by_K.div(a.by_splits.div(rest, split), kvh);
    RowTile t;
    t.tok0 = (long long)cache * a.c.tokens;
    t.head0 = (int)kvh * a.c.gq;
    t.R = a.c.tokens * a.c.gq;
    t.r0 = (int)tile * ST_ROWS;
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
    const KvSpan& sn = a.s;
    // Of the tile's tokens that see anything: the largest and the least count, the first and the last first row.
    int most = 0, low = 0x7fffffff, first = 0x7fffffff, late = 0;
    {
        const int last = (int)a.c.by_gq.div((uint32_t)min(t.r0 + ST_ROWS, t.R) - 1);
        for (int k = (int)a.c.by_gq.div((uint32_t)t.r0) + lane; k <= last; k += 32) {
            const int n = min(a.c.own.len[t.tok0 + k], a.c.own.rows);
            if (n <= 0) continue;
            const int w = span_first(sn, n);
            most = max(most, n);
            low = min(low, n);
            first = min(first, w);
            late = max(late, w);
        }
        most = __reduce_max_sync(0xffffffffu, most);
        low = __reduce_min_sync(0xffffffffu, low);
        first = __reduce_min_sync(0xffffffffu, first);
        late = __reduce_max_sync(0xffffffffu, late);
    }
    const SpanBlocks<ST_KEYS> blocks(sn, most, first);
    // This block's key blocks; none where they are fewer than the splits: the part then weighs nothing.
    const int blk0 = (int)((long long)split * blocks.count / a.splits);
    const int nb = (int)((long long)(split + 1) * blocks.count / a.splits) - blk0;
    // Key (value) block i into its ring slot (bf16).
    auto load = [&](bool is_v, int i) {
        const int sl = i % NS;
        uint64_t* full = (is_v ? vfull : kfull) + sl;
        uint8_t* base = stages + sl * L::STAGE + (is_v ? L::KVBYTES : 0);
        ptx::mbar_expect_tx(full, (uint32_t)L::KVBYTES);
        for (int db = 0; db < NDB; ++db)
            kv_load_box(base + db * (ST_KEYS * 128), is_v ? &maps.v : &maps.k, full, db * 64, a.at, (int)kvh, blocks.row(blk0 + i), cache);
    };
    if (warp == 0 && ptx::elect_one()) {
        if (!Q8) {
            ptx::prefetch_tmap(&maps.k);
            ptx::prefetch_tmap(&maps.v);
        }
        for (int b = 0; b < NB; ++b) {
            ptx::mbar_init(&sfull[b], 1);
            ptx::mbar_init(&pfull[b], ST_SOFT);
            ptx::mbar_init(&odone[b], 1);
        }
        for (int b = 0; b < NG; ++b) ptx::mbar_init(&gdone[b], 1);
        ptx::mbar_init(alldone, 1);
        ptx::mbar_init(qready, 256);
        for (int s = 0; s < NS; ++s) {
            ptx::mbar_init(&kfull[s], Q8 ? ST_CONV / 2 : 1);
            ptx::mbar_init(&vfull[s], Q8 ? ST_CONV / 2 : 1);
            ptx::mbar_init(&kempty[s], 1);
            ptx::mbar_init(&vempty[s], 1);
        }
        ptx::fence_mbar_init();
        *flag = 0;
        for (int b = 0; b < NG; ++b) begun[b] = 0;
    }
    if (warp == 1) {
        ptx::tmem_alloc(tmem_slot, L::TMEM_COLS);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp <= 1) {
        if (!Q8 && ptx::elect_one()) {
            const bool is_v = warp == 1;
            uint64_t* fullb = is_v ? vfull : kfull;
            uint64_t* emptyb = is_v ? vempty : kempty;
            int issued = 0;
            bool good = true;
            for (int i = 0; i < nb; ++i) {
                if (i >= NS) good = ptx::mbar_wait_bounded(&emptyb[i % NS], (i / NS - 1) & 1, ST_WAIT_NS);
                // (the query rows pass through the last value slots)
                else if (is_v && i >= NS - L::QS) good = ptx::mbar_wait_bounded(qready, 0, ST_WAIT_NS);
                if (!good) break;
                load(is_v, i);
                issued = i + 1;
            }
            if (!good) *flag = DEV_TIMEOUT_WEIGHTS;
            if (!ptx::ring_drain(fullb, NS, issued, ST_WAIT_NS)) *flag = DEV_TIMEOUT_WEIGHTS;
        }
    } else if (warp == 2) {
        if (ptx::elect_one()) {
            const uint32_t sb = ptx::smem_u32(stages);
            bool good = ptx::mbar_wait_bounded(qready, 0, ST_WAIT_NS);
            for (int i = 0; i < nb; ++i) {
                const int sl = i % NS;
                // (its score buffer holds P_{i-NB} until that product is done)
                if (i >= NB && good) good = ptx::mbar_wait_bounded(&odone[i % NB], (i / NB - 1) & 1, ST_WAIT_NS);
                if (good) good = ptx::mbar_wait_bounded(&kfull[sl], (i / NS) & 1, ST_WAIT_NS);
                ptx::tc_fence_after();
                if (good) {
                    const uint64_t kb = ptx::desc_sw128(sb + sl * L::STAGE);
#pragma unroll
                    for (int db = 0; db < NDB; ++db)
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            ptx::mma_bf16_ta(tmem + (uint32_t)(ST_KEYS * (i % NB)), tmem + L::TMEM_Q + (uint32_t)(8 * (4 * db + kk)),
                                             ptx::desc_add(kb, db * (ST_KEYS * 128) + kk * 32), IDESC_S, (db | kk) != 0);
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
                if (good) good = ptx::mbar_wait_bounded(&pfull[i % NB], (i / NB) & 1, ST_WAIT_NS);
                if (good) good = ptx::mbar_wait_bounded(&vfull[sl], (i / NS) & 1, ST_WAIT_NS);
                ptx::tc_fence_after();
                if (good) {
                    const uint64_t vb = ptx::desc_sw128_mn(sb + sl * L::STAGE + L::KVBYTES, ST_KEYS * 128, 1024);
#pragma unroll
                    for (int kk = 0; kk < ST_KEYS / 16; ++kk)
                        ptx::mma_bf16_ta(tmem + L::TMEM_O + (uint32_t)(i % NG * DP), tmem + (uint32_t)(ST_KEYS * (i % NB) + 8 * kk),
                                         ptx::desc_add(vb, kk * 16 * 128), IDESC_PV, i >= NG || kk != 0 || begun[i % NG] != 0);
                }
                if (i + NS < nb) ptx::mma_commit(&vempty[sl]);
                if (i + NB < nb) ptx::mma_commit(&odone[i % NB]);
                if (i + NG < nb) ptx::mma_commit(&gdone[i % NG]);
            }
            ptx::mma_commit(alldone);
            if (!good) *flag = DEV_TIMEOUT_MMA;
        }
    } else if (Q8 && tid >= L::CONV) {
        // Codes to fp16 numbers in the layout of the copies: 16 codes of a row are two 16-byte chunks of a 128-byte line. Each thread
        // copies pieces of its own ahead, and waits for no other's. Rows that no query row sees arrive as zeros.
        constexpr int PIECES = DP / 16, HALFT = ST_CONV / 2, MINE = ST_KEYS * PIECES / HALFT, SWEEP = HALFT / PIECES;   // rows of a sweep
        const bool is_v = tid >= L::CONV + HALFT;
        // Eight lanes are four pieces of a 128-byte line in two rows, whose chunks lie in eight places of the banks.
        const int x = (tid - L::CONV) % HALFT, piece = (x & 3) | (x >> 3) % (PIECES / 4) << 2, row0 = (x >> 2 & 1) + 2 * ((x >> 3) / (PIECES / 4));
        uint64_t* fullb = is_v ? vfull : kfull;
        uint64_t* emptyb = is_v ? vempty : kempty;
        const bool in = 16 * piece < a.c.D;
        const uint8_t* src = static_cast<const uint8_t*>(is_v ? a.c.own.v : a.c.own.k) + cache * a.c.own.cs + kvh * a.c.own.hs + (in ? 16 * piece : 0);
        uint8_t* const raw = st_smem + L::RING + is_v * (L::RAWBYTES / 2) + x * 16;
        auto fetch = [&](int i) {
            if (i < nb) {
                const int key0 = blocks.row(blk0 + i);
                const uint32_t to = ptx::smem_u32(raw + i % L::RAW * L::RAWBYTES);
                const bool all = key0 + ST_KEYS <= most && (key0 >= first || key0 + ST_KEYS <= sn.sink);
                const uint8_t* p = src + (key0 + row0) * a.c.own.rs;
#pragma unroll
                for (int m = 0; m < MINE; ++m) {
                    const bool live = in && (all || span_sees(sn, key0 + row0 + m * SWEEP, most, first));
                    ptx::cp_async_16(to + m * (HALFT * 16), live ? p : src, live);
                    p += SWEEP * a.c.own.rs;
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        bool good = true;
#pragma unroll
        for (int i = 0; i < L::RAW - 1; ++i) fetch(i);
        for (int i = 0; i < nb; ++i) {
            const int sl = i % NS;
            fetch(i + L::RAW - 1);
            if (good && i >= NS) good = ptx::mbar_wait_bounded(&emptyb[sl], (i / NS - 1) & 1, ST_WAIT_NS);
            // (the query rows pass through the last value slots)
            if (good && is_v && i >= NS - L::QS && i < NS) good = ptx::mbar_wait_bounded(qready, 0, ST_WAIT_NS);
            if (!good) break;
            asm volatile("cp.async.wait_group %0;" ::"n"(L::RAW - 1) : "memory");
            // Chunk c of row r lies at c ^ (r & 7) of its line; a sweep is four rows, or a multiple of eight.
            static_assert(SWEEP == 4 || SWEEP % 8 == 0, "rows of a sweep");
            uint8_t* base = stages + sl * L::STAGE + (is_v ? L::KVBYTES : 0) + piece / 4 * (ST_KEYS * 128) + row0 * 128;
            const uint32_t place = (uint32_t)((2 * (piece & 3)) ^ (row0 & 7)) << 4;
#pragma unroll
            for (int m = 0; m < MINE; ++m) {
                const uint4 c = *reinterpret_cast<const uint4*>(raw + i % L::RAW * L::RAWBYTES + m * (HALFT * 16));
                uint8_t* line = base + m * (SWEEP * 128);
                const uint32_t at = place ^ (uint32_t)((m * SWEEP & 7) << 4);
                *reinterpret_cast<uint4*>(line + at) = make_uint4(kv8_half2(c.x), kv8_half2(c.x >> 16), kv8_half2(c.y), kv8_half2(c.y >> 16));
                *reinterpret_cast<uint4*>(line + (at ^ 16)) = make_uint4(kv8_half2(c.z), kv8_half2(c.z >> 16), kv8_half2(c.w), kv8_half2(c.w >> 16));
            }
            ptx::fence_proxy_async_smem();
            ptx::mbar_arrive(&fullb[sl]);
        }
        ptx::cp_async_wait_all();   // (nothing may land once the block has left)
        if (!good) *flag = DEV_TIMEOUT_WEIGHTS;
    } else {
        const int grp = (warp - 4) >> 3, row = (warp & 3) * 32 + lane, half = ((warp - 4) >> 2) & 1;
        const int r = t.r0 + row;
        const bool valid = r < t.R;
        const int vis = valid ? min(max(a.c.own.len[row_token(a.c, t, r)], 0), a.c.own.rows) : 0;   // the row's count
        const int begins = span_first(sn, vis);
        const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t out = lane_base + L::TMEM_O + (uint32_t)(grp * DP);
        const uint32_t pair_bar = 1 + 4 * grp + (warp & 3);   // the two warps of these 32 rows
        float m_used = -INFINITY, l = 0.f;          // m_used is the same in both threads of a row
        int v_used = ST_NONE;                       // 8 bits: the largest scale of values that the row has seen; likewise
        bool good = true;
        // The query rows were loaded 128 bytes of four rows an instruction: through 4 KB of shared memory of the warp
        // to a row per thread, then to TMEM (column 32 db + 4 c + e holds elements 64 db + 8 c + 2 e, + 1).
        if (grp == 0) {
            const int wi = warp - 4;
            float qf[8];   // 8 bits: what row 4 i + lane / 8 is multiplied by
            if constexpr (Q8) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float top = 0.f;
#pragma unroll
                    for (int k = 0; k < QN; ++k) {
                        const uint32_t w[4] = {qv[k][i].x, qv[k][i].y, qv[k][i].z, qv[k][i].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float lo = fabsf(__uint_as_float(w[e] << 16)), hi = fabsf(__uint_as_float(w[e] & 0xffff0000u));
                            top = fmaxf(top, lo < INFINITY ? lo : 0.f);
                            top = fmaxf(top, hi < INFINITY ? hi : 0.f);
                        }
                    }
#pragma unroll
                    for (int e = 1; e < 8; e <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, e));
                    if ((lane & 7) == 0) qmax[half * ST_ROWS + (warp & 3) * 32 + 4 * i + (lane >> 3)] = top;
                }
                ptx::named_bar_sync(pair_bar, 64);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int rr = (warp & 3) * 32 + 4 * i + (lane >> 3);
                    const float top = fmaxf(qmax[rr], qmax[ST_ROWS + rr]);
                    qf[i] = kv8_pow2(255 - max((int)(__float_as_uint(top) >> 23), 2));   // the largest to 2 .. 4
                }
            }
            uint4* turn = (uint4*)(stages + (NS - 1 - wi / L::TURN) * L::STAGE + L::KVBYTES + wi % L::TURN * 4096);
#pragma unroll
            for (int k = 0; k < QN; ++k) {
                const int db = half + 2 * k;
                if (db < NDB) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint4 v = qv[k][i];
                        if constexpr (Q8) {
                            uint32_t* w = &v.x;
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                w[e] = half_pair(__uint_as_float(w[e] << 16) * qf[i], __uint_as_float(w[e] & 0xffff0000u) * qf[i]);
                        }
                        turn[(4 * i + (lane >> 3)) * 8 + ((lane & 7) ^ ((4 * i + (lane >> 3)) & 7))] = v;
                    }
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
        constexpr int HK = ST_KEYS / 2;   // keys per thread
        // In 8 bits scores are those of the scaled query, qs of them the true ones; maxima are those of the scores in log2 units, with their
        // keys' scales (a score times either factor alone may pass fp32's range).
        float qs = 1.f;
        if constexpr (Q8) {
            if (grp > 0) good = ptx::mbar_wait_bounded(qready, 0, ST_WAIT_NS);
            qs = kv8_pow2(max((int)(__float_as_uint(fmaxf(qmax[row], qmax[ST_ROWS + row])) >> 23), 2) - 1);
        }
        const float c2s = fminf(a.c2 * qs, 3e38f);
        const uint64_t c2 = pair2(c2s);
        const float unit = Q8 ? 1.f : c2s;   // log2 units of a maximum's
        const float rescale = Q8 ? ST_RESCALE8 : fminf(ST_RESCALE / c2s, 3e38f);
        // Scales of the group's next blocks, a byte a thread (of a tile that no row sees: 127).
        uint8_t* const sc = st_smem + L::SC_OFF + grp * ST_RUN * 8;
        auto scales = [&](int i0) {
            const int e = (tid - 128) % ST_SOFT, i = i0 + e / 8 * NG;
            static_assert(ST_RUN * 8 == ST_SOFT, "one byte a thread");
            uint8_t byte = 127;
            if (i < nb) {
                const int at = blocks.row(blk0 + i) + 16 * (e & 3);
                if (at < most && (at < sn.sink || at + 16 > first))
                    byte = (e & 4 ? sn.vs : sn.ks)[((long long)cache * a.c.K + kvh) * sn.nblk + (at >> sn.n_log2)];
            }
            ptx::named_bar_sync(11 + grp, ST_SOFT);   // the last ones have been read
            sc[e] = byte;
            ptx::named_bar_sync(11 + grp, ST_SOFT);
        };
        for (int i = grp; i < nb; i += NG) {
            uint2 by = make_uint2(0, 0);   // 8 bits: scales of the block's tiles, keys' and values'
            if constexpr (Q8) {
                const int k = i / NG % ST_RUN;
                if (k == 0) scales(i);
                by = *(const uint2*)(sc + 8 * k);
            }
            if (good) good = ptx::mbar_wait_bounded(&sfull[i % NB], (i / NB) & 1, ST_WAIT_NS);
            ptx::tc_fence_after();
            uint32_t s[2][16];
            {
                const uint32_t sa = lane_base + (uint32_t)(ST_KEYS * (i % NB) + HK * half);
                ptx::tmem_ld_x16(sa, s[0]);
                ptx::tmem_ld_x16(sa + 16u, s[1]);
                ptx::tmem_ld_wait();
            }
            const int key0 = blocks.row(blk0 + i), mine = key0 + HK * half;
            // Of this half's keys the ones that the row sees: all, or those below `end`, from `from` on or below `sunk`.
            const int end = vis - mine, from = begins - mine, sunk = sn.sink - mine;
            const bool full = __all_sync(0xffffffffu, end >= HK && (from <= 0 || sunk >= HK));
            auto sees = [&](int j) { return j < end && (j >= from || j < sunk); };
            if (!full) {
#pragma unroll
                for (int j = 0; j < HK; ++j)
                    if (!sees(j)) s[j >> 4][j & 15] = __float_as_uint(-INFINITY);
            }
            float mt[2] = {-INFINITY, -INFINITY};   // of the half's tiles
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int j = 0; j < 16; ++j) m4[j & 3] = fmaxf(m4[j & 3], __uint_as_float(s[e][j]));
                mt[e] = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            }
            // 8 bits: scores are the products times the scale of their tile's keys, which is in what scores and maximum are multiplied by.
            float kc[2] = {c2s, c2s};
            if constexpr (Q8) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t k = by.x >> (16 * half + 8 * e) & 255u;
                    if (k == 255) {   // NaN: so are the scores of those that see them
#pragma unroll
                        for (int j = 0; j < 16; ++j) s[e][j] = sees(16 * e + j) ? 0x7fffffffu : __float_as_uint(-INFINITY);
                        mt[e] = -INFINITY;
                    } else {
                        kc[e] = fminf(fmaxf(c2s * kv8_scale(k), 0x1p-126f), 3e38f);   // (0 times a hidden score would be NaN, as infinity times 0)
                        mt[e] *= kc[e];
                    }
                }
            }
            float mb = fmaxf(mt[0], mt[1]);
            float* xm = xmax + (2 * grp + (i / NG & 1)) * 2 * ST_ROWS + row;
            xm[half * ST_ROWS] = mb;
            ptx::named_bar_sync(pair_bar, 64);
            mb = fmaxf(mb, xm[(1 - half) * ST_ROWS]);
            const bool move = mb - m_used > rescale;   // (of -infinities NaN: no)
            const float alpha = !move ? 1.f : m_used == -INFINITY ? 0.f : kr_ex2((m_used - mb) * unit);
            float beta = alpha;               // what the outputs are multiplied by: in units of the largest scale, too
            bool grown = false;
            float pv[2] = {1.f, 1.f};         // what the probabilities of the half's tiles are multiplied by
            uint32_t nan = 0;                 // tiles of the half whose values are NaN
            if constexpr (Q8) {
                int v_now = v_used;
                uint32_t top = __vmaxu4(by.y & 0xffff, by.y >> 16);
                top = max(top & 255, top >> 8);
                if (__any_sync(0xffffffffu, (int)top > v_used)) {   // (else no row has to look)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int at = key0 + 16 * e, v = by.y >> (8 * e) & 255;
                        if (v != 255 && at < vis && (at < sn.sink || at + 16 > begins)) v_now = max(v_now, max(v, 1));
                    }
                }
                grown = v_now != v_used;
                if (grown) beta *= kv8_pow2(127 + v_used - v_now);
                v_used = v_now;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = by.y >> (16 * half + 8 * e) & 255;
                    if (at == 255) nan |= 1u << e;
                    pv[e] = at == 255 || v_now == ST_NONE ? (float)(1 << ST_BOOST) : kv8_pow2(min(127 + ST_BOOST + at - v_now, 254));
                }
            }
            // TMEM accesses are warp-collective: the warp rescales together (its half of the columns), lanes whose
            // maximum stays put multiply by 1. O is settled once P V of the group's previous block is done.
            if (__any_sync(0xffffffffu, i >= NG && ((move && m_used != -INFINITY) || grown))) {
                if (good) good = ptx::mbar_wait_bounded(&gdone[grp], (i / NG - 1) & 1, ST_WAIT_NS);
                ptx::tc_fence_after();
#pragma unroll 1
                for (int c0 = half * (DP / 2); c0 < (half + 1) * (DP / 2); c0 += 32) {
                    uint32_t ro[2][16];
                    ptx::tmem_ld_x16(out + (uint32_t)c0, ro[0]);
                    ptx::tmem_ld_x16(out + (uint32_t)(c0 + 16), ro[1]);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) ro[j >> 4][j & 15] = __float_as_uint(__uint_as_float(ro[j >> 4][j & 15]) * beta);
                    ptx::tmem_st_x16(out + (uint32_t)c0, ro[0]);
                    ptx::tmem_st_x16(out + (uint32_t)(c0 + 16), ro[1]);
                }
                ptx::tmem_st_wait();
            }
            if (move) {
                l *= alpha;
                m_used = mb;
            }
            // 2^((s - m) c): a hidden key's -inf gives 0, also while the row has seen none at all (m taken as 0).
            const float m_now = m_used == -INFINITY ? 0.f : m_used;
            const uint64_t neg_m = pair2(-m_now), k2[2] = {pair2(kc[0]), pair2(kc[1])};   // (k2: 8 bits)
            float l4[4] = {0.f, 0.f, 0.f, 0.f};
            uint32_t pk[HK / 2];
#pragma unroll
            for (int k = 0; k < HK; k += 2) {
                float p0, p1;
                if constexpr (Q8) {
                    // (as a product and a sum in one rounding the maximum's own would be what its rounding left: above 2^27 much more than 0)
                    scale_sub2(__uint_as_float(s[k >> 4][k & 15]), __uint_as_float(s[k >> 4][(k + 1) & 15]), k2[k >> 4], m_now, p0, p1);
                } else {
                    sub_scale2(__uint_as_float(s[k >> 4][k & 15]), __uint_as_float(s[k >> 4][(k + 1) & 15]), neg_m, c2, p0, p1);
                }
                p0 = kr_ex2(p0);
                p1 = kr_ex2(p1);
                l4[(k >> 1) & 3] += p0 + p1;
                pk[k / 2] = Q8 ? half_pair(p0 * pv[k >> 4], p1 * pv[k >> 4]) : kr_pack(p0, p1);
            }
            // Values under a scale that is NaN are NaN to the rows that see them, by way of their probabilities.
            if (Q8 && nan) {
#pragma unroll
                for (int k = 0; k < HK; ++k)
                    if ((nan >> (k >> 4) & 1) && sees(k)) pk[k / 2] |= k & 1 ? 0x7fff0000u : 0x7fffu;
            }
            l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
            // Keys of the block that some row sees and some does not; rows that none sees. The same for all threads.
            const bool cut = max(key0, low) < min(key0 + ST_KEYS, most) || max(max(key0, sn.sink), first) < min(key0 + ST_KEYS, late);
            const bool dead = most < key0 + ST_KEYS || (key0 < first && key0 + ST_KEYS > sn.sink);
            uint8_t* vb = stages + i % NS * L::STAGE + L::KVBYTES;
            if (cut) {
                // Is there an infinity or NaN among the values?
                if (good) good = ptx::mbar_wait_bounded(&vfull[i % NS], (i / NS) & 1, ST_WAIT_NS);
                uint32_t top = 0;   // the largest magnitudes, 16 bits each
#pragma unroll
                for (int e0 = 0; e0 < ST_KEYS * NDB * 8; e0 += ST_SOFT) {
                    const int e = e0 + (tid - 128) % ST_SOFT, key = e / (NDB * 8), p = e % (NDB * 8);
                    uint4 v = *(const uint4*)(vb + (p / 8) * (ST_KEYS * 128) + key * 128 + (p % 8) * 16);
                    if (!span_sees(sn, key0 + key, most, first)) v = make_uint4(0, 0, 0, 0);
                    top = __vmaxu2(__vmaxu2(top, v.x & 0x7fff7fffu), v.y & 0x7fff7fffu);
                    top = __vmaxu2(__vmaxu2(top, v.z & 0x7fff7fffu), v.w & 0x7fff7fffu);
                }
                constexpr uint32_t INF = Q8 ? 0x7c00u : 0x7f80u;
                if (group_any(11 + grp, ST_SOFT, (top & 0xffffu) >= INF || top >> 16 >= INF)) {
                    // Row by row: first one half's keys, then the other's, onto the settled output of the blocks before.
                    if (i >= NG && good) good = ptx::mbar_wait_bounded(&gdone[grp], (i / NG - 1) & 1, ST_WAIT_NS);
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
                                    if (!sees(k)) continue;
                                    const int key = HK * half + k;
                                    float pr;
                                    if (Q8) pr = __half2float(__ushort_as_half((unsigned short)(k & 1 ? pk[k / 2] >> 16 : pk[k / 2])));
                                    else pr = __uint_as_float(k & 1 ? pk[k / 2] & 0xffff0000u : pk[k / 2] << 16);
                                    const uint8_t* vr = vb + (c0 / 64) * (ST_KEYS * 128) + key * 128;
#pragma unroll
                                    for (int h = 0; h < 2; ++h) {
                                        const uint4 v = *(const uint4*)(vr + (((c0 % 64 / 8 + h) ^ (key & 7)) << 4));
                                        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                        for (int e = 0; e < 4; ++e) {
                                            uint32_t &y0 = ro[8 * h + 2 * e], &y1 = ro[8 * h + 2 * e + 1];
                                            float2 z = make_float2(__uint_as_float(x[e] << 16), __uint_as_float(x[e] & 0xffff0000u));
                                            if (Q8) z = __half22float2(*reinterpret_cast<const __half2*>(&x[e]));
                                            y0 = __float_as_uint(fmaf(pr, z.x, __uint_as_float(y0)));
                                            y1 = __float_as_uint(fmaf(pr, z.y, __uint_as_float(y1)));
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
                    ptx::named_bar_sync(11 + grp, ST_SOFT);   // every thread has read the values
                    for (int e = (tid - 128) % ST_SOFT; good && e < ST_KEYS * NDB * 8; e += ST_SOFT) ((uint4*)vb)[e] = make_uint4(0, 0, 0, 0);
                    if (i < NG && tid % ST_SOFT == 128) begun[grp] = 1;
                    ptx::fence_proxy_async_smem();
                }
            }
            // Over the scores of both halves: both threads of a row have read theirs (the barrier above). Column 16 half
            // + e holds keys 32 half + 2 e, + 1.
            ptx::tmem_st_x16(lane_base + (uint32_t)(ST_KEYS * (i % NB) + 16 * half), pk);
            ptx::tmem_st_wait();
            if (!Q8 && dead) {
                // Values of rows that no row sees, as they landed: cleared (a row's 16-byte pieces stay in the row).
                if (good) good = ptx::mbar_wait_bounded(&vfull[i % NS], (i / NS) & 1, ST_WAIT_NS);
#pragma unroll
                for (int e0 = 0; e0 < ST_KEYS * NDB * 8; e0 += ST_SOFT) {
                    const int e = e0 + (tid - 128) % ST_SOFT, key = e / (NDB * 8), p = e % (NDB * 8);
                    if (good && !span_sees(sn, key0 + key, most, first))
                        *(uint4*)(vb + (p / 8) * (ST_KEYS * 128) + key * 128 + (p % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                ptx::fence_proxy_async_smem();
            }
            ptx::tc_fence_before();
            ptx::mbar_arrive(&pfull[i % NB]);
        }
        // The row's sum: both halves, in order, through the buffer that the last block's maxima are not in.
        const int mine = (nb - grp + NG - 1) / NG;   // blocks of this group
        float* xl = xmax + (2 * grp + (mine & 1)) * 2 * ST_ROWS + row;
        xl[half * ST_ROWS] = l;
        ptx::named_bar_sync(pair_bar, 64);
        l = xl[0] + xl[ST_ROWS];
        // Every P V of the block is done, and with them every read of the ring.
        if (good) good = ptx::mbar_wait_bounded(alldone, 0, ST_WAIT_NS);
        ptx::tc_fence_after();
        if (!good) *flag = DEV_TIMEOUT_MMA;
        // The groups' sums are joined, and their outputs on the way: w_g = 2^((m_g - M) c), nothing of a group in which the row saw no
        // key.
        float w = 1.f;
        const bool some = l != 0.f;
        if (NG > 1) {
            if (half == 0) ml[grp * ST_ROWS + row] = make_float2(m_used, l);
            ptx::named_bar_sync(9, NG * ST_SOFT);
            const float2 other = ml[(1 - grp) * ST_ROWS + row];
            const float M = fmaxf(m_used, other.x);
            w = m_used == -INFINITY ? 0.f : kr_ex2((m_used - M) * unit);
            l = w * l + (other.x == -INFINITY ? 0.f : kr_ex2((other.x - M) * unit)) * other.y;   // (0 times a NaN sum is NaN)
            m_used = M;
        }
        float vscale = 1.f;
        if constexpr (Q8) {
            m_used *= 1.f / a.c2;
            w *= 1.f / (1 << ST_BOOST);
            vscale = v_used == ST_NONE ? 1.f : kv8_scale((uint32_t)v_used);
        }
        // A result is scaled by 1 / l and rounded on its way.
        const float inv = l == 0.f ? 0.f : 1.f / l;   // (0: the row saw no key; a NaN score makes l, and so the row, NaN)
        uint8_t* orow = st_smem + row * L::OUT_LD;
        // A half row's 16-bit values go where its own 32-bit ones were.
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
                    if (good && nb > 0) {
                        uint4 packed;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            uint4* dst = (uint4*)(orow + (c0 + 4 * k) * 4);
                            float x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                x[e] = __uint_as_float(v[k >> 2][4 * (k & 3) + e]);
                                x[e] = some ? w * x[e] : 0.f;
                                if (Q8) x[e] *= vscale;
                            }
                            if (grp > 0) {
                                const uint4 y = *dst;
                                x[0] += __uint_as_float(y.x);
                                x[1] += __uint_as_float(y.y);
                                x[2] += __uint_as_float(y.z);
                                x[3] += __uint_as_float(y.w);
                            }
                            if (a.out && grp == NG - 1) {   // 16 bytes for every two of these
                                uint32_t* p = (k & 1) ? &packed.z : &packed.x;
                                p[0] = kr_pack(x[0] * inv, x[1] * inv);
                                p[1] = kr_pack(x[2] * inv, x[3] * inv);
                                if (k & 1) *(uint4*)(orow + half * (DP * 2) + (c0 + 4 * (k - 1) - half * (DP / 2)) * 2) = packed;
                            } else {
                                *dst = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
                            }
                        }
                    }
                }
            }
            if (turn + 1 < NG) ptx::named_bar_sync(10, NG * ST_SOFT);
        }
        if (grp == NG - 1 && half == 0 && valid) {
            const long long row_at = row_index(a.c, t, r);
            if constexpr (JOIN) ml[row] = make_float2(m_used, l);   // (the groups' have been read)
            else if (!a.out) a.pml[row_at * a.splits + split] = make_float2(m_used, l);
            else if (a.lse) a.lse[row_at] = l == 0.f ? -INFINITY : fmaf(m_used, a.c.scale, logf(l));
        }
        // Rows leave by whole warps. (A bulk copy a row, 128 of them, took 3 thousand cycles longer.)
        ptx::named_bar_sync(9, NG * ST_SOFT);
        if constexpr (!JOIN) {
#pragma unroll 4
            for (int rr = warp - 4; rr < ST_ROWS; rr += 8 * NG) {
                if (!good || t.r0 + rr >= t.R) continue;
                const long long row_at = row_index(a.c, t, t.r0 + rr);
                const uint8_t* from = st_smem + rr * L::OUT_LD;
                if (a.out) {
                    const int d = 8 * lane, h = d >= DP / 2;
                    if (d < a.c.D)
                        *(uint4*)(a.out + row_at * a.c.D + d) = nb == 0 ? make_uint4(0, 0, 0, 0) : *(const uint4*)(from + h * (DP * 2) + (d - h * (DP / 2)) * 2);
                } else if (nb > 0) {
                    for (int d = 4 * lane; d < a.c.D; d += 128)
                        *(uint4*)(a.po + ((long long)split * a.rows + row_at) * a.c.D + d) = *(const uint4*)(from + 4 * d);
                }
            }
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    // Before the pair meets: another block's allocation may wait for these columns, and its partner for that one.
    if (warp == 1) ptx::tmem_dealloc(tmem, L::TMEM_COLS);
    if constexpr (JOIN) {
        // The parts of the tile are in the shared memories of the cluster's blocks, each of which writes some of the rows.
        ptx::cluster_sync_all();
        bool whole = true;
        for (int k = 0; k < ST_RANKS; ++k) whole = whole && __float_as_int(ptx::dsmem_ld_f32(ptx::dsmem_map(ptx::smem_u32(flag), (uint32_t)k))) == 0;
        if (whole) join_tile<DP, L::OUT_LD, L::THREADS / 32>(a, t, (int)split, st_smem, ml, tid >> 5, lane);
        __syncwarp();
        ptx::cluster_sync_all();   // every block's rows have been read
    }
    if (tid == 0 && *flag != 0) atomicCAS(a.err, 0, *flag);
}

template <int DP>
jpi_status launch_dim(const SpanTileArgs& a, const SpanMaps& m, unsigned blocks, cudaStream_t st) {
    auto* const kernel = a.s.ks ? (a.joined ? k_kv_span_t5<DP, true, true> : k_kv_span_t5<DP, true, false>)
                                : (a.joined ? k_kv_span_t5<DP, false, true> : k_kv_span_t5<DP, false, false>);
    return kv_start_clusters(kernel, dim3(blocks), a.joined ? ST_RANKS : 1, a.s.ks ? StSmem<DP, true>::THREADS : StSmem<DP, false>::THREADS,
                             (size_t)(a.s.ks ? StSmem<DP, true>::BYTES : StSmem<DP, false>::BYTES), false, st, m, a);
}

template <int DP>
jpi_status prepare_dim(jpi_kv_handle* h) {
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_span_t5<DP, false, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, StSmem<DP, false>::BYTES));
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_span_t5<DP, true, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, StSmem<DP, true>::BYTES));
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_span_t5<DP, false, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, StSmem<DP, false>::BYTES));
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_span_t5<DP, true, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, StSmem<DP, true>::BYTES));
    JPI_TRY(kv_resident_clusters(k_kv_span_t5<DP, false, true>, ST_RANKS, StSmem<DP, false>::THREADS, StSmem<DP, false>::BYTES, &h->tile_pairs[0]));
    return kv_resident_clusters(k_kv_span_t5<DP, true, true>, ST_RANKS, StSmem<DP, true>::THREADS, StSmem<DP, true>::BYTES, &h->tile_pairs[1]);
}

// Rows of the cache that the tokens of a tile see at most.
long long tile_span(const KvCall& c, const KvSpan& s) {
    const long long toks = std::min<long long>(c.tokens, (ST_ROWS + c.gq - 1) / c.gq + 1);
    return std::min<long long>(c.own.rows, (long long)s.window + toks + std::min(s.sink, c.own.rows) + ST_KEYS);
}

}  // namespace

jpi_status kv_span_tiles_prepare(jpi_kv_handle* h) {
    if (!h->bf16 || h->D < 64) return JPI_OK;
    return h->D <= 64 ? prepare_dim<64>(h) : h->D <= 128 ? prepare_dim<128>(h) : prepare_dim<256>(h);
}

int kv_span_tiles_plan(const jpi_kv_handle* h, const KvCall& c, const KvSpan& s, long long room, bool* joined) {
    *joined = false;
    if (!h->bf16 || c.D < 64 || h->tiles == 0) return 0;
    const long long R = (long long)c.tokens * c.gq, tiles = (R + ST_ROWS - 1) / ST_ROWS, blocks = tiles * c.K * c.batch;
    const long long span = tile_span(c, s), nb = (span + ST_KEYS - 1) / ST_KEYS;
    KvMapDims m;
    if (!s.ks && !kv_map_dims(c.own, c.K, c.D, c.batch, &m)) return 0;
    if (blocks * nb >= 1ll << 31) return 0;
    if (h->tiles < 0 && (R < ST_LEAST || (R + KR_ROWS - 1) / KR_ROWS * c.K * c.batch * span * c.D <= st_row_elements(s.ks, R, c.D))) return 0;
    // Splits by which the waves of blocks end first; a result in parts has its combine, and its rows to and from the workspace, or, of two
    // parts in clusters that are all resident together, their meeting. (In clusters of four the meeting takes what the combine does: 64
    // tokens of 8 heads over 2100 keys of 256 17.2 us for 15.5.)
    long long best = 1, best_time = -1;
    for (long long n = 1; n <= std::min(nb, std::max(1ll, 2ll * h->num_sms / blocks)); ++n) {
        const bool meet = n == ST_RANKS && blocks <= h->tile_pairs[s.ks != nullptr];
        if (!meet && n > room) continue;
        const long long time = (blocks * n + h->num_sms - 1) / h->num_sms * ((nb + n - 1) / n * st_block(s.ks, c.D) + ST_ENDS) +
                               (meet ? st_meet(c.D) : n > 1 ? ST_JOIN + 2 * n * c.batch * c.tokens * c.H * c.D * 4 / ST_BYTES : 0);
        if (best_time < 0 || time < best_time) {
            best_time = time;
            best = n;
            *joined = meet;
        }
    }
    return (int)best;
}

jpi_status launch_kv_span_tiles(jpi_kv_handle* h, const KvCall& c, const KvSpan& s, int splits, bool joined, float* po, float2* pml, void* out,
                                float* lse, cudaStream_t st) {
    SpanTileArgs a = {};
    SpanMaps maps = {};
    a.c = c;
    a.s = s;
    a.c2 = KR_LOG2E * c.scale;
    a.splits = splits;
    a.tiles = (int)(((long long)c.tokens * c.gq + ST_ROWS - 1) / ST_ROWS);
    a.by_splits = KvDiv((uint32_t)a.splits);
    a.by_tiles = KvDiv((uint32_t)a.tiles);
    a.by_rest = KvDiv((uint32_t)((long long)splits * c.K * c.batch));
    a.tiles_outer = (long long)c.batch * c.K * c.own.rows * c.D * (s.ks ? 2 : 4) <= 64ll << 20;
    a.po = po;
    a.pml = pml;
    a.rows = (long long)c.batch * c.tokens * c.H;
    a.out = splits == 1 ? static_cast<__nv_bfloat16*>(out) : nullptr;
    a.joined = joined ? static_cast<__nv_bfloat16*>(out) : nullptr;
    if (joined) a.tiles_outer = true;   // (a cluster's blocks are the splits of one tile)
    a.lse = lse;
    a.err = h->dev_err;
    if (!s.ks) {
        KvMapDims m;
        if (!kv_map_dims(c.own, c.K, c.D, c.batch, &m) || !kv_make_map(m, c.own.k, c.D, ST_KEYS, &maps.k) ||
            !kv_make_map(m, c.own.v, c.D, ST_KEYS, &maps.v)) {
            set_error("cuTensorMapEncodeTiled refused the cache");
            return JPI_ERR_CUDA;
        }
        a.at = make_int3(m.at_head, m.at_row, m.at_cache);
    }
    const unsigned blocks = (unsigned)((long long)a.tiles * splits * c.K * c.batch);
    return c.D <= 64 ? launch_dim<64>(a, maps, blocks, st) : c.D <= 128 ? launch_dim<128>(a, maps, blocks, st) : launch_dim<256>(a, maps, blocks, st);
}

}  // namespace jpi
