// Attention of a batch over shared prefixes and own rows (jpi_kv_attend).
//
//   o_r = sum_j p_rj v_j,  p_rj = exp(s_rj - lse_r),  s_rj = scale q_r . k_j,
// j over the first prefix_len rows of the run's prefix and then the first `seen` rows of the request's own
// cache. A prefix is read once for all its requests: their query rows are one matrix.
//
// The softmax is computed in parts: every part (a range of keys of one side) keeps a running maximum m and
// sum l per row and an unnormalised output, all fp32, and they are joined as
//   o = sum_s w_s O_s / sum_s w_s l_s,  w_s = exp(scale (m_s - M)),
// in part order, so that a result does not depend on which block finished first. A part that saw no key
// has l = 0 and weighs nothing; a row of only such parts is zero, its lse -inf. (m = -inf is no sign of it: maxima skip
// NaN, and a part whose scores are all NaN has m = -inf and l = NaN. l alone says which, and a NaN l makes the whole row
// NaN, its lse too, whatever the other parts hold.) Maxima are those of the unscaled
// products, and the difference is scaled, not the product: log2(e) times a score near the type's largest
// values would overflow.
//
// Kernels: the row kernels here take both sides, 8 query rows a warp; a side with many query rows on the same keys
// goes to tiles of 128 rows instead (kv_attend_t5.cu) where the call is large, bound by tensor cores and 2^x where the row kernel is
// bound by memory, so the two share the SMs: the row kernel starts first with two blocks per SM, the tiles start while it
// runs. k_kv_combine joins the parts, except where a row has only one.

#include "kv_parts.cuh"
#include "kv_attend.h"

#include <algorithm>

namespace jpi {
namespace {

// Joins elements d0 .. d0 + DP - 1 of parts first, first + step, .. of a row (of `parts`) to `r`, which holds nothing yet,
// relative to their largest maximum. The loads of JOIN parts are in flight together: they are made whether the part holds
// anything or not (its memory is the workspace's), and a part of no keys, which was never written, is replaced by zeros.
template <int DP>
__device__ __forceinline__ void join_parts(const AttendArgs& a, RowAcc<DP>& r, long long row, int d0, int first, int step, int lane) {
    constexpr int NI = RowAcc<DP>::NI, JOIN = 16 / NI;
    const float2* pml = a.pml + row * a.parts;
    int d[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) d[i] = d0 + 4 * lane + 128 * i < a.c.D ? d0 + 4 * lane + 128 * i : 0;
    const int mine = (a.parts - first + step - 1) / step;   // parts of this warp
    for (int p0 = 0; p0 < mine; p0 += 32) {
        const int n = min(32, mine - p0);
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < n) ml = __ldcg(pml + first + (p0 + lane) * step);
        float M = fmaxf(r.m, ml.x);
#pragma unroll
        for (int e = 16; e > 0; e >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, e));
        const float w0 = r.m == -INFINITY ? 0.f : kr_ex2((r.m - M) * a.c2);
        const float w = ml.x == -INFINITY ? 0.f : kr_ex2((ml.x - M) * a.c2);
        const uint32_t written = __ballot_sync(0xffffffffu, lane < n && ml.y != 0.f);
        float l = w * ml.y;
#pragma unroll
        for (int e = 16; e > 0; e >>= 1) l += __shfl_xor_sync(0xffffffffu, l, e);
        r.l = r.l * w0 + l;
        r.m = M;
#pragma unroll
        for (int i = 0; i < NI; ++i) r.o[i] = make_float4(r.o[i].x * w0, r.o[i].y * w0, r.o[i].z * w0, r.o[i].w * w0);
        for (int k0 = 0; k0 < n; k0 += JOIN) {
            float4 v[JOIN][NI];
            float wk[JOIN];
#pragma unroll
            for (int k = 0; k < JOIN; ++k) {
                const int q = min(k0 + k, n - 1);
                const float* src = a.po + ((first + (p0 + q) * step) * a.rows + row) * a.c.D;
                wk[k] = __shfl_sync(0xffffffffu, w, q);
                if (k0 + k >= n) wk[k] = 0.f;
#pragma unroll
                for (int i = 0; i < NI; ++i) v[k][i] = __ldcg((const float4*)(src + d[i]));
            }
#pragma unroll
            for (int k = 0; k < JOIN; ++k) {
#pragma unroll
                for (int i = 0; i < NI; ++i)
                    if (k0 + k >= n || !(written >> (k0 + k) & 1)) v[k][i] = make_float4(0.f, 0.f, 0.f, 0.f);
                r.add(wk[k], v[k]);
            }
        }
    }
}

// bf16. A warp works alone: it takes pieces (8 query rows over a range of keys) in turn and streams their blocks of 16
// (D to 256) to 64 (D to 64) keys, 16 KB with their values, through two stages of shared memory of its own by 16-byte
// asynchronous copies, the next piece's first blocks and query rows behind this one's last. So a piece has no start-up
// of its own and pieces can be small enough to even out requests of different lengths; what is in flight needs neither
// registers nor room in L1; and rows that no query of the piece sees arrive as zeros.
//
// Keys are the 16 rows of mma.sync m16n8k16 and query rows its 8 columns; the values' product runs over keys with
// d as its rows, so that the probabilities turn from one's result into the other's operand by 8 x 8 transposes within
// the warp. Probabilities enter that product as two bf16 terms (the rounded value and what the rounding left), so that
// its error stays that of fp32 sums: the kernel is bound by memory, not by its products.
constexpr int RT_STAGE = 16384;

template <int DP>
struct RtSmem {
    static constexpr int KEYS = RT_STAGE / (4 * DP);     // keys of a block
    static constexpr int HALF = RT_STAGE / 2;            // its keys' bytes; its values follow
    static constexpr int QBYTES = KR_ROWS * DP * 2;      // query rows of a piece: two pieces' worth
    static constexpr int Q_OFF = 2 * RT_STAGE;
    static constexpr int SEEN_OFF = Q_OFF + 2 * QBYTES;  // [AHEAD][8] counts of the pieces in hand
    static constexpr int AHEAD = 4;
    static constexpr int BYTES = SEEN_OFF + AHEAD * KR_ROWS * 4;
    static constexpr int BESIDE = DP == 256 ? 2 : DP == 128 ? 3 : 4;   // blocks that fit beside the tiles on an SM
    static constexpr int ALONE = DP == 256 ? 5 : 6;                    // and without them
    // A warp beside the tiles has the registers that theirs leave in its quarter of the SM's file.
    static constexpr int REGS = DP == 256 ? 224 : 152;
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}

template <int DP>
__global__ void __maxnreg__(RtSmem<DP>::REGS) k_kv_attend_rows(const __grid_constant__ AttendArgs a) {
    using L = RtSmem<DP>;
    extern __shared__ __align__(128) uint8_t rt_smem[];
    constexpr int MT = L::KEYS / 16;   // 16-key tiles of a block
    constexpr int ND = DP / 16;
    constexpr int CH = DP / 8;         // 16-byte chunks of a row; chunk c of row r lies at c ^ (r & 7)
    constexpr int RPI = 32 / CH > 0 ? 32 / CH : 1;   // rows one instruction of the warp copies
    const int lane = threadIdx.x, g = lane >> 2, j = lane & 3;
    const uint32_t sm = ptx::smem_u32(rt_smem);
    int* const counts = (int*)(rt_smem + L::SEEN_OFF);
    ptx::grid_dep_launch();
    const uint32_t pieces = (uint32_t)(a.p.blocks + a.o.blocks);
    const int D = a.c.D, mych = lane % CH, myrow = lane / CH;
    const bool dlive = 8 * mych < D;
    const float slack = 8.f / a.c2;

    // ---- what is to be copied: pieces opened in order, block by block
    uint32_t f_piece = blockIdx.x;   // the next piece to open
    int f_seq = 0, f_full = 0, f_blk = 0, f_end = 0, f_lim = 0;   // f_full: opened pieces that have blocks
    const __nv_bfloat16 *f_k = nullptr, *f_v = nullptr;   // this lane's chunk of the open piece's row 0
    long long f_rs = 0;
    int ahead = 0;                   // this lane's row's count of the next piece (lanes 0-7), on its way since the last one opened
    auto peek = [&]() {
        ahead = 0;
        if (f_piece < pieces) {
            const Piece x = piece_of(a, f_piece, 0);
            if (lane < KR_ROWS) ahead = row_seen(a.c, x.prefix, x.cache, x.t, x.t.r0 + lane);
        }
    };
    int issued = 0, used = 0;        // blocks asked for, and through
    int seq = 0, full = 0;           // pieces finished, and begun with blocks
    // Asks for the next block, opening pieces on the way (at most AHEAD in hand); false if there is none.
    auto produce = [&]() {
        while (f_blk >= f_end) {
            if (f_piece >= pieces || f_seq - seq >= L::AHEAD) return false;
            const Piece x = piece_of(a, f_piece, 0);
            const SidePlan& sp = x.prefix ? a.p : a.o;
            const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
            if (lane < KR_ROWS) counts[(f_seq & (L::AHEAD - 1)) * KR_ROWS + lane] = ahead;
            f_lim = __reduce_max_sync(0xffffffffu, lane < KR_ROWS ? ahead : 0);
            const int nb = (f_lim + L::KEYS - 1) / L::KEYS;
            f_blk = (int)((long long)nb * x.split / sp.splits);
            f_end = (int)((long long)nb * (x.split + 1) / sp.splits);
            if (f_blk < f_end) {
                const long long base = x.cache * s.cs + x.kvh * s.hs + (dlive ? 8 * mych : 0);
                f_k = static_cast<const __nv_bfloat16*>(s.k) + base;
                f_v = static_cast<const __nv_bfloat16*>(s.v) + base;
                f_rs = s.rs;
                // The query rows travel with the first block. (Two pieces' fit: with two blocks in hand, the piece with
                // blocks before the last one is through.)
#pragma unroll
                for (int i = 0; i < KR_ROWS / RPI; ++i) {
                    const int rr = i * RPI + myrow, r = x.t.r0 + rr;
                    const bool in = dlive && r < x.t.R;
                    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.c.q) + (in ? row_query(a.c, x.t, r) + 8 * mych : 0);
                    ptx::cp_async_16(sm + L::Q_OFF + (f_full & 1) * L::QBYTES + rr * (DP * 2) + ((mych ^ (rr & 7)) << 4), q, in);
                }
                ++f_full;
            }
            ++f_seq;
            f_piece += gridDim.x;
            peek();
        }
        const uint32_t dst = sm + (issued & 1) * RT_STAGE;
        const int key0 = f_blk * L::KEYS;
        const __nv_bfloat16 *k = f_k + (long long)(key0 + myrow) * f_rs, *v = f_v + (long long)(key0 + myrow) * f_rs;
#pragma unroll
        for (int i = 0; i < L::KEYS / RPI; ++i) {
            const int rr = i * RPI + myrow;
            const bool in = dlive && key0 + rr < f_lim;
            const uint32_t at = rr * (DP * 2) + ((mych ^ (rr & 7)) << 4);
            ptx::cp_async_16(dst + at, in ? k : f_k, in);
            ptx::cp_async_16(dst + L::HALF + at, in ? v : f_v, in);
            k += RPI * f_rs;
            v += RPI * f_rs;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ++issued;
        ++f_blk;
        return true;
    };

    peek();
    if (produce()) produce();
    for (uint32_t piece = blockIdx.x; piece < pieces; piece += gridDim.x, ++seq) {
        const Piece x = piece_of(a, piece, 0);
        const SidePlan& sp = x.prefix ? a.p : a.o;
        if (f_seq <= seq) produce();   // (opens it, if the pieces before had fewer blocks than there are stages)
        __syncwarp();
        // What the lane's rows 2 j, 2 j + 1 see, and the most and the least of the tile's rows.
        const int n0 = counts[(seq & (L::AHEAD - 1)) * KR_ROWS + 2 * j], n1 = counts[(seq & (L::AHEAD - 1)) * KR_ROWS + 2 * j + 1];
        const int rj = x.t.r0 + 2 * j;
        int lim = max(n0, n1), low = min(rj < x.t.R ? n0 : 0x7fffffff, rj + 1 < x.t.R ? n1 : 0x7fffffff);
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            lim = max(lim, __shfl_xor_sync(0xffffffffu, lim, o));
            low = min(low, __shfl_xor_sync(0xffffffffu, low, o));
        }
        const int nb = (lim + L::KEYS - 1) / L::KEYS;
        const int b0 = (int)((long long)nb * x.split / sp.splits), b1 = (int)((long long)nb * (x.split + 1) / sp.splits);
        uint32_t qf[ND][2];
        float o[ND][4];
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        for (int blk = b0; blk < b1; ++blk) {
            const int key0 = blk * L::KEYS;
            if (issued == used) produce();
            // This block's copies have landed; the one after may be on its way.
            if (issued - used > 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
            const uint32_t ks = sm + (used & 1) * RT_STAGE, vs = ks + L::HALF;
            if (blk == b0) {
                const uint32_t qs = sm + L::Q_OFF + (full++ & 1) * L::QBYTES + (lane & 7) * (DP * 2);
#pragma unroll
                for (int i = 0; i < ND; i += 2) {
                    uint32_t f[4];
                    ldsm4(f, qs + (((2 * i + (lane >> 3)) ^ (lane & 7)) << 4));
                    qf[i][0] = f[0];
                    qf[i][1] = f[1];
                    qf[i + 1][0] = f[2];
                    qf[i + 1][1] = f[3];
                }
            }
            // Four chains of products whatever the shape: one of D / 16 steps would be its latency.
            constexpr int NCH = MT >= 4 ? 1 : 4 / MT;
            float part[NCH][MT][4];
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[c][t][e] = 0.f;
            const int kr = (lane & 7) + (lane & 8);   // key of this lane's matrix row; its chunk is 2 i + lane / 16
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    uint32_t f[4];
                    ldsm4(f, ks + (16 * t + kr) * (DP * 2) + (((2 * i + (lane >> 4)) ^ (kr & 7)) << 4));
                    kr_mma(part[i % NCH][t], f[0], f[1], f[2], f[3], qf[i][0], qf[i][1]);
                }
            float sc[MT][4];
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sc[t][e] = part[0][t][e];
#pragma unroll
                    for (int c = 1; c < NCH; ++c) sc[t][e] += part[c][t][e];
                }
            // Keys g, g + 8 of each tile, rows 2 j, 2 j + 1; hidden scores are replaced, whatever they hold.
            const bool cut = low < key0 + L::KEYS;   // the same for the warp
            if (cut) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = key0 + 16 * t + g + 8 * e;
                        if (key >= n0) sc[t][2 * e] = -INFINITY;
                        if (key >= n1) sc[t][2 * e + 1] = -INFINITY;
                    }
            }
            float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    x0 = fmaxf(x0, sc[t][2 * e]);
                    x1 = fmaxf(x1, sc[t][2 * e + 1]);
                }
            // The maximum moves only when a score passes it by more than 8 in log2 units (probabilities stay below 2^8):
            // most blocks do not, and need no maximum over the keys' lanes.
            if (__any_sync(0xffffffffu, x0 > m0 + slack || x1 > m1 + slack)) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, d));
                    x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, d));
                }
                const float y0 = fmaxf(m0, x0), y1 = fmaxf(m1, x1);
                const float a0 = m0 == -INFINITY ? 0.f : kr_ex2((m0 - y0) * a.c2);
                const float a1 = m1 == -INFINITY ? 0.f : kr_ex2((m1 - y1) * a.c2);
                m0 = y0;
                m1 = y1;
                l0 *= a0;
                l1 *= a1;
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    o[i][0] *= a0;
                    o[i][1] *= a1;
                    o[i][2] *= a0;
                    o[i][3] *= a1;
                }
            }
            const float f0 = m0 == -INFINITY ? 0.f : m0, f1 = m1 == -INFINITY ? 0.f : m1;
            uint32_t ph[MT][2], pe[MT][2];
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float p0 = kr_ex2((sc[t][2 * e] - f0) * a.c2), p1 = kr_ex2((sc[t][2 * e + 1] - f1) * a.c2);
                    l0 += p0;
                    l1 += p1;
                    const uint32_t h = kr_pack(p0, p1);
                    const uint32_t r = kr_pack(p0 - __uint_as_float(h << 16), p1 - __uint_as_float(h & 0xffff0000u));
                    ph[t][e] = kr_transpose(h);
                    pe[t][e] = kr_transpose(r);
                }
            const int vr = (lane & 7) + ((lane >> 4) << 3);   // key of this lane's matrix row; its chunk is 2 i + bit 3
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    uint32_t f[4];
                    ldsm4_t(f, vs + (16 * t + vr) * (DP * 2) + (((2 * i + ((lane >> 3) & 1)) ^ (vr & 7)) << 4));
                    kr_mma(o[i], f[0], f[1], f[2], f[3], ph[t][0], ph[t][1]);
                    kr_mma(o[i], f[0], f[1], f[2], f[3], pe[t][0], pe[t][1]);
                }
            __syncwarp();   // every lane has read the stage
            ++used;
            produce();
        }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        // An infinite value times what the rounding left of its probability (0, or of the other sign) is NaN, and so is 0 times an
        // infinity or NaN that only another row of the tile sees. Rows whose sum is finite and outputs are not are formed
        // again, key by key in fp32, each over its own keys. (One check a piece, where a search of every block that some rows see a
        // part of would read its values twice.)
        float z0 = 0.f, z1 = 0.f;   // 0 as long as all are finite
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            z0 = fmaf(o[i][0], 0.f, fmaf(o[i][2], 0.f, z0));
            z1 = fmaf(o[i][1], 0.f, fmaf(o[i][3], 0.f, z1));
        }
        uint32_t again = __reduce_or_sync(0xffffffffu, (rj < x.t.R && l0 < INFINITY && !(z0 == 0.f) ? 1u << (2 * j) : 0u) |
                                                           (rj + 1 < x.t.R && l1 < INFINITY && !(z1 == 0.f) ? 2u << (2 * j) : 0u));
        for (; again; again &= again - 1) {
            const int r = __ffs(again) - 1;
            const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
            const int n = min(b1 * L::KEYS, __shfl_sync(0xffffffffu, (r & 1) ? n1 : n0, r >> 1));
            float m = __shfl_sync(0xffffffffu, (r & 1) ? m1 : m0, r >> 1);
            if (m == -INFINITY) m = 0.f;
            constexpr int NL = DP / 32;   // lane's elements of a row: lane + 32 i
            const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.c.q) + row_query(a.c, x.t, x.t.r0 + r);
            const long long base = x.cache * s.cs + x.kvh * s.hs;
            float qr[NL], sum[NL];
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                qr[i] = lane + 32 * i < D ? __bfloat162float(q[lane + 32 * i]) : 0.f;
                sum[i] = 0.f;
            }
#pragma unroll 1
            for (int key = b0 * L::KEYS; key < n; ++key) {
                const __nv_bfloat16 *k = static_cast<const __nv_bfloat16*>(s.k) + base + key * s.rs,
                                    *v = static_cast<const __nv_bfloat16*>(s.v) + base + key * s.rs;
                float dot = 0.f;
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    if (lane + 32 * i < D) dot = fmaf(qr[i], __bfloat162float(k[lane + 32 * i]), dot);
#pragma unroll
                for (int e = 16; e > 0; e >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, e);
                const float pr = kr_ex2((dot - m) * a.c2);
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    if (lane + 32 * i < D) sum[i] = fmaf(pr, __bfloat162float(v[lane + 32 * i]), sum[i]);
            }
            // Back to the fragments: elements 16 i + g, + 8 of the row to the lanes of its column.
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                const float y0 = __shfl_sync(0xffffffffu, sum[i >> 1], 16 * (i & 1) + g), y1 = __shfl_sync(0xffffffffu, sum[i >> 1], 16 * (i & 1) + g + 8);
                if (r == 2 * j) o[i][0] = y0, o[i][2] = y1;
                if (r == 2 * j + 1) o[i][1] = y0, o[i][3] = y1;
            }
        }
        // Rows 2 j (elements 0 and 2 of each fragment) and 2 j + 1 (1 and 3), d = 16 i + g and + 8.
        const bool in0 = rj < x.t.R, in1 = rj + 1 < x.t.R;
        const long long row0 = in0 ? row_index(a.c, x.t, rj) : 0, row1 = in1 ? row_index(a.c, x.t, rj + 1) : 0;
        if (a.out) {
            // The only part: the result itself. Lanes g and g + 1 exchange halves, so that the even one has a pair of row
            // 2 j and the odd one a pair of row 2 j + 1.
            const bool even = (g & 1) == 0;
            const float inv0 = inverse_sum(l0), inv1 = inverse_sum(l1);
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + (even ? row0 : row1) * D + (g & ~1);
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float u = o[i][2 * e] * inv0, v = o[i][2 * e + 1] * inv1;
                    const float w = __shfl_xor_sync(0xffffffffu, even ? v : u, 4);
                    if ((even ? in0 : in1) && 16 * i + 8 * e < D)
                        *(uint32_t*)(out + 16 * i + 8 * e) = even ? kr_pack(u, w) : kr_pack(w, v);
                }
            if (g == 0 && a.lse) {
                if (in0) a.lse[row0] = log_sum(m0, l0, a.c.scale);
                if (in1) a.lse[row1] = log_sum(m1, l1, a.c.scale);
            }
        } else {
            const long long at0 = x.part * a.rows + row0, at1 = x.part * a.rows + row1;
            if (g == 0 && in0) a.pml[row0 * a.parts + x.part] = make_float2(m0, l0);
            if (g == 0 && in1) a.pml[row1 * a.parts + x.part] = make_float2(m1, l1);
            float *o0 = a.po + at0 * D + g, *o1 = a.po + at1 * D + g;
            const bool w0 = in0 && l0 != 0.f, w1 = in1 && l1 != 0.f;
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (16 * i + 8 * e >= D) continue;
                    if (w0) o0[16 * i + 8 * e] = o[i][2 * e];
                    if (w1) o1[16 * i + 8 * e] = o[i][2 * e + 1];
                }
        }
    }
}

// fp32 on CUDA cores: one warp = 8 query rows over 32-key blocks. Scores with a key per lane, the values with a lane per four
// elements of d. What bounds it is latency: a block's loads, its products (5 instructions for 4 of them) and 2^x follow one
// another in a warp, and a small call has a block or two per warp. So the loads of several pieces of a key are on their way
// together, those of the next values while these are used, in as many registers as leave an SM three blocks, and a warp with
// its keys to itself writes its rows from registers: 4 requests of 9 tokens over 342 keys took 20 us with loads one by one, 16
// with 8 at a time, 14 so; a call of 294 tokens over 103 keys 54, 36 and 37 (44 with two blocks an SM).
template <int DP>
__global__ void __launch_bounds__(AT_THREADS, DP == 256 ? 2 : 3) k_kv_attend_f32(const __grid_constant__ AttendArgs a) {
    extern __shared__ __align__(16) float kv_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    ptx::grid_dep_launch();
    const Piece x = piece_of(a, blockIdx.x, warp);
    const SidePlan& sp = x.prefix ? a.p : a.o;
    const KvSide& s = x.prefix ? a.c.prefix : a.c.own;
    const int D = a.c.D;
    float* qs = kv_smem + warp / sp.wk * (KR_ROWS * DP);
    const int wk = warp % sp.wk;
    if (wk == 0) {
        for (int e0 = lane; e0 < KR_ROWS * (DP / 4); e0 += 4 * 32) {
            float4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = e0 + 32 * i, r = x.t.r0 + e / (DP / 4), d = 4 * (e % (DP / 4));
                v[i] = r < x.t.R && d < D ? *(const float4*)(static_cast<const float*>(a.c.q) + row_query(a.c, x.t, r) + d)
                                          : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) *(float4*)(qs + 4 * (e0 + 32 * i)) = v[i];
        }
    }
    int n[KR_ROWS], lim = 0;
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r) {
        n[r] = row_seen(a.c, x.prefix, x.cache, x.t, x.t.r0 + r);
        lim = max(lim, n[r]);
    }
    __syncthreads();
    const long long nb = (lim + 31) / 32;
    const int b0 = (int)(nb * x.split / sp.splits), b1 = (int)(nb * (x.split + 1) / sp.splits);
    const float* kbase = (const float*)s.k + x.cache * s.cs + (x.kvh) * s.hs;
    const float* vbase = (const float*)s.v + x.cache * s.cs + (x.kvh) * s.hs;
    constexpr int NI = (DP + 127) / 128;
    constexpr int KL = 4 / NI, VL = 4 / NI;   // 16-byte loads of a key, values, that are on their way at a time
    float4 o[KR_ROWS][NI];
    float m[KR_ROWS], l[KR_ROWS];
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) o[r][i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int blk = b0 + wk; blk < b1; blk += sp.wk) {
        const int key0 = blk * 32, key = key0 + lane;
        float p[KR_ROWS];
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) p[r] = 0.f;
        const float* kp = kbase + (long long)key * s.rs;
        // Values of VL keys, those of the next ones on their way while these are used, the first ones during the scores.
        float4 next[VL][NI];
        auto load = [&](int t0) {
#pragma unroll
            for (int t = 0; t < VL; ++t)
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int d = 4 * lane + 128 * i;
                    next[t][i] = d < D && key0 + t0 + t < lim ? __ldg((const float4*)(vbase + (long long)(key0 + t0 + t) * s.rs + d))
                                                              : make_float4(0.f, 0.f, 0.f, 0.f);
                }
        };
        load(0);
        for (int d0 = 0; d0 < D; d0 += 4 * KL) {
            float4 k[KL];
#pragma unroll
            for (int i = 0; i < KL; ++i)
                k[i] = key < lim && d0 + 4 * i < D ? __ldg((const float4*)(kp + d0 + 4 * i)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                if (d0 + 4 * i >= D) break;
#pragma unroll
                for (int r = 0; r < KR_ROWS; ++r) {
                    const float4 q = *(const float4*)(qs + r * DP + d0 + 4 * i);
                    p[r] = fmaf(q.x, k[i].x, fmaf(q.y, k[i].y, fmaf(q.z, k[i].z, fmaf(q.w, k[i].w, p[r]))));
                }
            }
        }
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) {
            const float sc = key < n[r] ? p[r] : -INFINITY;
            float mx = sc;
#pragma unroll
            for (int e = 16; e > 0; e >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, e));
            if (mx > m[r]) {
                const float al = m[r] == -INFINITY ? 0.f : exp2f((m[r] - mx) * a.c2);
                m[r] = mx;
                l[r] *= al;
#pragma unroll
                for (int i = 0; i < NI; ++i) o[r][i] = make_float4(o[r][i].x * al, o[r][i].y * al, o[r][i].z * al, o[r][i].w * al);
            }
            p[r] = exp2f((sc - (m[r] == -INFINITY ? 0.f : m[r])) * a.c2);   // (of -inf 0, of NaN NaN)
            l[r] += p[r];
        }
        for (int t0 = 0; t0 < 32 && key0 + t0 < lim; t0 += VL) {
            float4 v[VL][NI];
#pragma unroll
            for (int t = 0; t < VL; ++t)
#pragma unroll
                for (int i = 0; i < NI; ++i) v[t][i] = next[t][i];
            if (t0 + VL < 32) load(t0 + VL);
#pragma unroll
            for (int t = 0; t < VL; ++t)
#pragma unroll
                for (int r = 0; r < KR_ROWS; ++r) {
                    const float w = __shfl_sync(0xffffffffu, p[r], t0 + t);
                    if (key0 + t0 + t < n[r]) {   // a hidden value is not even multiplied by zero
#pragma unroll
                        for (int i = 0; i < NI; ++i) {
                            o[r][i].x = fmaf(w, v[t][i].x, o[r][i].x);
                            o[r][i].y = fmaf(w, v[t][i].y, o[r][i].y);
                            o[r][i].z = fmaf(w, v[t][i].z, o[r][i].z);
                            o[r][i].w = fmaf(w, v[t][i].w, o[r][i].w);
                        }
                    }
                }
        }
    }
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r)
#pragma unroll
        for (int e = 16; e > 0; e >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], e);
    if (sp.wk == 1) {   // (of the whole block) nothing to merge
#pragma unroll
        for (int r = 0; r < KR_ROWS; ++r) {
            if (x.t.r0 + r >= x.t.R) break;
            const long long row = row_index(a.c, x.t, x.t.r0 + r);
            if (a.out) {
                RowAcc<DP> acc;
                acc.m = m[r];
                acc.l = l[r];
#pragma unroll
                for (int i = 0; i < NI; ++i) acc.o[i] = o[r][i];
                write_row<DP, float>(a, acc, row, 0, lane);
                continue;
            }
            if (lane == 0) a.pml[row * a.parts + x.part] = make_float2(m[r], l[r]);
            if (l[r] == 0.f) continue;
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (4 * lane + 128 * i < D) *(float4*)(a.po + (x.part * a.rows + row) * D + 4 * lane + 128 * i) = o[r][i];
        }
        return;
    }
    __syncthreads();   // the queries have been read
    float* f = kv_smem + warp * MergeSmem<DP>::WARP_FLOATS;
#pragma unroll
    for (int r = 0; r < KR_ROWS; ++r) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int d = 4 * lane + 128 * i;
            if (d < DP) *(float4*)(f + r * MergeSmem<DP>::LD + d) = o[r][i];
        }
        if (lane == 0) {
            f[KR_ROWS * MergeSmem<DP>::LD + 2 * r] = m[r];
            f[KR_ROWS * MergeSmem<DP>::LD + 2 * r + 1] = l[r];
        }
    }
    merge_and_write<DP, float>(a, x, sp, kv_smem, warp, lane);
}

// Joins the parts of all rows, DP elements of one (from DP blockIdx.y on) by `wpr` warps (a power of two), each with every
// wpr-th part, then the warps in order. Latency bounds it: 16 loads of a lane are on their way together, and where the rows are few
// a row of more than 128 elements is two blocks'. (One request over 65536 keys, 760 parts of 256 elements, took 28 us with
// both halves in one warp and 25 so; 48 requests of 32 heads with 30011 shared keys 58 with up to four warps a row and 55
// with as many as are resident together; 16 x 10 tokens of 8 heads in 2 parts 11.1 with the halves apart, 9.6 together.)
constexpr int CB_WARPS = 16;   // most of a block
template <int DP, typename E>
__global__ void __launch_bounds__(32 * CB_WARPS) k_kv_combine(const __grid_constant__ AttendArgs a, int wpr) {
    __shared__ float4 so[CB_WARPS][RowAcc<DP>::NI][32];
    __shared__ float2 sml[CB_WARPS];
    constexpr int NI = RowAcc<DP>::NI;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = warp & (wpr - 1), d0 = DP * blockIdx.y;
    const long long row = ((long long)blockIdx.x * (blockDim.x >> 5) + warp) / wpr;
    ptx::grid_dep_wait();
    RowAcc<DP> acc;
    acc.m = -INFINITY;
    acc.l = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) acc.o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < a.rows) join_parts<DP>(a, acc, row, d0, first, wpr, lane);
    if (wpr > 1) {
#pragma unroll
        for (int i = 0; i < NI; ++i) so[warp][i][lane] = acc.o[i];
        if (lane == 0) sml[warp] = make_float2(acc.m, acc.l);
        __syncthreads();
        if (first != 0) return;
        float M = acc.m;
        for (int k = 1; k < wpr; ++k) M = fmaxf(M, sml[warp + k].x);
        acc.m = M;
        acc.l = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) acc.o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < wpr; ++k) {
            const float2 ml = sml[warp + k];
            const float w = ml.x == -INFINITY ? 0.f : kr_ex2((ml.x - M) * a.c2);
            float4 v[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) v[i] = so[warp + k][i][lane];
            acc.add(w, v);
            acc.l += w * ml.y;
        }
    }
    if (row < a.rows) write_row<DP, E>(a, acc, row, d0, lane);
}

// A side's pieces for blocks of `warps` warps, whose warps take `step` keys at a time. Key splits: up to `want` pieces
// in all while a warp keeps `least` keys (below that a part's rows are as many bytes as a good share of its keys); but a
// call of few pieces is split down to single steps, as far as two blocks an SM go: it is waited for (one request over 816
// and 40 keys: 8.5 us by single steps, 8.6 by two, 9.5 by three). The parts fit their
// half of the workspace.
SidePlan plan_side(const jpi_kv_handle* h, const KvCall& c, bool prefix, int warps, int step, int least, long long want) {
    SidePlan s;
    const KvSide& side = prefix ? c.prefix : c.own;
    if (side.rows == 0) return s;
    const int caches = prefix ? c.groups : c.batch;
    const long long R = (long long)(prefix ? c.batch / c.groups : 1) * c.tokens * c.gq;
    const long long rt = (R + KR_ROWS - 1) / KR_ROWS;
    while (s.wr < warps && s.wr < rt) s.wr *= 2;
    s.wk = warps / s.wr;
    s.tiles = (int)((rt + s.wr - 1) / s.wr);
    const long long blocks = (long long)caches * c.K * s.tiles, rows = (long long)c.batch * c.tokens * c.H;
    const long long room = std::max(1ll, (ws_rows(h) / 2) / rows);
    const long long coarse = std::min(want / blocks, ((long long)side.rows + least * s.wk - 1) / (least * s.wk));
    const long long fine = std::min(2ll * h->num_sms / blocks, ((long long)side.rows + step * s.wk - 1) / (step * s.wk));
    s.splits = (int)std::max(1ll, std::min(std::max(coarse, fine), room));
    s.blocks = blocks * s.splits;
    s.by_splits = KvDiv((uint32_t)s.splits);
    s.by_tiles = KvDiv((uint32_t)s.tiles);
    return s;
}

template <int DP>
jpi_status launch_dim(jpi_kv_handle* h, const KvCall& c, void* out, float* lse, cudaStream_t st) {
    AttendArgs a = {};
    a.c = c;
    a.c2 = KR_LOG2E * c.scale;
    a.rows = (long long)c.batch * c.tokens * c.H;
    a.po = static_cast<float*>(h->ws);
    a.pml = reinterpret_cast<float2*>(a.po + (size_t)ws_rows(h) * c.D);
    a.lse = lse;
    KvTilesPlan tiles;
    kv_tiles_plan(h, c, std::max(1ll, ws_rows(h) / 2 / a.rows), &tiles);
    const bool beside = tiles.takes(false) || tiles.takes(true);
    if (h->bf16) {
        // Single warps with 64 KB of keys and values or more each.
        constexpr int KEYS = RtSmem<DP>::KEYS;
        const long long want = (long long)(beside ? RtSmem<DP>::BESIDE : RtSmem<DP>::ALONE) * h->num_sms;
        a.p = plan_side(h, c, true, 1, KEYS, 4 * KEYS, want);
        a.o = plan_side(h, c, false, 1, KEYS, 4 * KEYS, want);
    } else {
        a.p = plan_side(h, c, true, AT_WARPS, 32, 32, 2ll * h->num_sms);
        a.o = plan_side(h, c, false, AT_WARPS, 32, 32, 2ll * h->num_sms);
    }
    for (int i = 0; i < 2; ++i)
        if (tiles.takes(i)) {
            SidePlan& s = i ? a.o : a.p;
            s.blocks = 0;
            s.splits = tiles.splits[i];
        }
    const int parts = a.parts = a.p.splits + a.o.splits;
    const long long pieces = a.p.blocks + a.o.blocks;
    if (pieces > 0x7fffffffll) {
        set_error("the call needs more than 2^31 blocks");
        return JPI_ERR_SHAPE;
    }
    if (pieces > 0) {
        AttendArgs r = a;
        if (parts == 1) r.out = out;
        if (h->bf16) {
            const long long most = (long long)(beside ? RtSmem<DP>::BESIDE : RtSmem<DP>::ALONE) * h->num_sms;
            JPI_TRY(kv_start(k_kv_attend_rows<DP>, std::min(pieces, most), 32, RtSmem<DP>::BYTES, false, st, r));
        } else {
            JPI_TRY(kv_start(k_kv_attend_f32<DP>, pieces, AT_THREADS, MergeSmem<DP>::BYTES, false, st, r));
        }
    }
    const int part0[2] = {0, a.p.splits};
    if (beside) JPI_TRY(launch_kv_tiles_t5(h, c, tiles, part0, a.po, a.pml, parts, out, lse, pieces > 0 && h->pdl, st));
    return parts == 1 ? JPI_OK : launch_kv_combine(h, c, parts, out, lse, st);
}

template <int DP>
jpi_status prepare_dim() {
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_f32<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, MergeSmem<DP>::BYTES));
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_rows<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, RtSmem<DP>::BYTES));
    // All of its loads go to shared memory, and the 128-row tiles need the SM set up for the most of it.
    JPI_CUDA_TRY(cudaFuncSetAttribute(k_kv_attend_rows<DP>, cudaFuncAttributePreferredSharedMemoryCarveout,
                                      cudaSharedmemCarveoutMaxShared));
    return JPI_OK;
}

}  // namespace

size_t kv_attend_ws_bytes(const jpi_kv_handle* h) {
    return (size_t)ws_rows(h) * (h->D * sizeof(float) + sizeof(float2));
}

jpi_status kv_attend_prepare(jpi_kv_handle* h) {
    JPI_TRY(kv_tiles_prepare(h));
    return h->D <= 64 ? prepare_dim<64>() : h->D <= 128 ? prepare_dim<128>() : prepare_dim<256>();
}

jpi_status launch_kv_combine(const jpi_kv_handle* h, const KvCall& c, int parts, void* out, float* lse, cudaStream_t st) {
    AttendArgs a = {};
    a.c = c;
    a.c2 = KR_LOG2E * c.scale;
    a.rows = (long long)c.batch * c.tokens * c.H;
    a.po = static_cast<float*>(h->ws);
    a.pml = reinterpret_cast<float2*>(a.po + (size_t)ws_rows(h) * c.D);
    a.parts = parts;
    a.out = out;
    a.lse = lse;
    // Warps for 8 to 16 parts each, to sixteen, as long as all are resident together (16 an SM).
    const int slices = c.D > 128 && a.rows * 2 <= 16ll * h->num_sms ? 2 : 1;
    int wpr = 1;
    while (wpr < CB_WARPS && wpr * 8 < parts && a.rows * slices * wpr * 2 <= 16ll * h->num_sms) wpr *= 2;
    const int warps = std::max(wpr, AT_WARPS);
    const dim3 grid((unsigned)((a.rows * wpr + warps - 1) / warps), (unsigned)slices);
    const bool wide = c.D > 128 && slices == 1;
    return kv_start(h->bf16 ? (wide ? k_kv_combine<256, __nv_bfloat16> : k_kv_combine<128, __nv_bfloat16>)
                            : (wide ? k_kv_combine<256, float> : k_kv_combine<128, float>), grid, 32 * warps, 0, h->pdl, st, a, wpr);
}

jpi_status launch_kv_attend(jpi_kv_handle* h, const KvCall& c, void* out, float* lse, cudaStream_t st) {
    return h->D <= 64 ? launch_dim<64>(h, c, out, lse, st)
                      : h->D <= 128 ? launch_dim<128>(h, c, out, lse, st) : launch_dim<256>(h, c, out, lse, st);
}

}  // namespace jpi
