// Eviction from a cache by accumulated attention weight (jpi_kv_evict): two launches, the choice and
// the move.
//
// The choice (k_kv_select), one block per layer, cache and KV head. The weights, as unsigned keys of
// the same order (NaN 0, below everything), are searched for the need-th largest by three passes over
// 11, 11 and 10 bits, a histogram in shared memory each: exact, whatever the distribution. Above the
// threshold every row stays; of the rows equal to it the lowest, as many as are left. Each warp has a
// run of consecutive rows (in registers up to 512), so that ballots and one sum over the warps give every row its place, the kept
// rows come out ascending and what a warp stores lies side by side (12 caches of 2513 rows: 10.6 us a call with a run per thread,
// 9.6 so). Its time is that of barriers and latencies, so every warp finds the bin by itself, from sums that all of them
// read: 8 barriers where a block-wide scan in each pass took 25 (18 caches of 816 rows 8.5 us a call, then 9.7). Of 16384
// rows half of its 17 us is the first read of the weights.
//
// The move (k_kv_gather): a block takes a slice (16 to 512 bytes, whole rows where there are blocks enough) of every
// kept row of one cache, head and matrix, in tiles of ascending rows: a tile is loaded whole, then stored. In place this
// needs no second buffer: a row never moves up (row i goes to at most i) and what a tile overwrites lies in it or
// before it, so it has been read. Apart, the tiles are independent and dealt to further blocks. Bound by memory: every
// kept row is read and written once.

#include "kv.h"
#include "../ptx.h"

#include <algorithm>

namespace jpi {
namespace {

constexpr int SEL_THREADS = 1024;
constexpr int SEL_BINS = 2048;

// An unsigned key of the same order; NaN is 0, -0 equals 0.
__device__ __forceinline__ uint32_t sort_key(float w) {
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Inclusive sums over the warp's lanes.
__device__ __forceinline__ uint32_t warp_scan(uint32_t x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}
// RUN: rows of a thread, their weights in registers; 0: any number, read again in every pass.
template <int RUN>
__global__ void __launch_bounds__(SEL_THREADS) k_kv_select(const float* w_all, const int* length, int rows, int caches,
                                                           int K, int keep, int sink, int recent, int dst_rows,
                                                           float* w_out_all, int* kept_all) {
    __shared__ __align__(8) uint32_t hist[3][SEL_BINS];      // of each pass, the largest digit first
    __shared__ uint32_t bin_sums[3][SEL_THREADS / 32];       // of 64 bins each
    __shared__ uint2 warp_sums[SEL_THREADS / 32];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    ptx::grid_dep_launch();
    const long long item = blockIdx.x;   // (layer, cache, head)
    const int c = (int)((item / K) % caches);
    const float* w = w_all + item * rows;
    float* w_out = w_out_all + item * dst_rows;
    int* kept = kept_all + item * keep;
    const int n = min(max(length[c], 0), rows);
    if (n <= keep) {
        for (int i = t; i < keep; i += SEL_THREADS) {
            kept[i] = i < n ? i : -1;
            if (i < n && w_out != w) w_out[i] = w[i];
        }
        return;
    }
    // A warp has 32 run consecutive rows, a lane every 32nd of them from `base` on.
    const int run = RUN > 0 ? RUN : (n + SEL_THREADS - 1) / SEL_THREADS, base = warp * 32 * run + lane;
    float ws[RUN > 0 ? RUN : 1];
    if constexpr (RUN > 0) {
#pragma unroll
        for (int e = 0; e < RUN; ++e) ws[e] = base + 32 * e < n ? w[base + 32 * e] : 0.f;
    }
    // f(row, key) for the thread's rows, and some past the end, by whole warps.
    auto each = [&](auto f) {
        if constexpr (RUN > 0) {
#pragma unroll
            for (int e = 0; e < RUN; ++e) f(base + 32 * e, sort_key(ws[e]));
        } else {
            for (int e = 0; e < run; ++e) f(base + 32 * e, base + 32 * e < n ? sort_key(w[base + 32 * e]) : 0u);
        }
    };
    // The need-th largest key of rows lo .. hi - 1 (need < hi - lo).
    const int lo = sink, hi = n - recent;
    uint32_t need = (uint32_t)(keep - sink - recent);
    uint32_t prefix = 0, mask = 0;   // keys with (key & mask) == prefix are still candidates
    if (need > 0) {
        const int shifts[3] = {21, 10, 0};
        for (int i = t; i < 3 * SEL_BINS; i += SEL_THREADS) hist[0][i] = 0;
        __syncthreads();
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = shifts[pass];
            const uint32_t last = pass == 2 ? 1023u : 2047u;   // the largest digit
            each([&](int i, uint32_t k) {
                if (i >= lo && i < hi && (k & mask) == prefix) atomicAdd(&hist[pass][last - ((k >> shift) & last)], 1u);
            });
            __syncthreads();
            // The bin that holds the need-th: each warp adds up 64 bins, then every warp finds the 64 and the bin by itself.
            const uint2 own = *(const uint2*)&hist[pass][64 * warp + 2 * lane];
            const uint32_t sum = __reduce_add_sync(0xffffffffu, own.x + own.y);
            if (lane == 0) bin_sums[pass][warp] = sum;
            __syncthreads();
            const uint32_t part = bin_sums[pass][lane], upto = warp_scan(part);
            const int seg = (__ffs(__ballot_sync(0xffffffffu, upto >= need)) - 1) & 31;   // (there is one)
            const uint32_t before = __shfl_sync(0xffffffffu, upto - part, seg);
            const uint2 two = *(const uint2*)&hist[pass][64 * seg + 2 * lane];
            const uint32_t in = before + warp_scan(two.x + two.y);
            const int at = (__ffs(__ballot_sync(0xffffffffu, in >= need)) - 1) & 31;
            const uint32_t above = __shfl_sync(0xffffffffu, in - two.x - two.y, at), first = __shfl_sync(0xffffffffu, two.x, at);
            const bool second = need > above + first;
            prefix |= (last - (uint32_t)(64 * seg + 2 * at + second)) << shift;
            mask |= last << shift;
            need -= second ? above + first : above;
        }
    }
    // Rows that stay: protected or above the threshold, and `need` of those equal to it.
    const bool some = keep > sink + recent;
    auto above = [&](int i, uint32_t k) { return i < n && (i < lo || i >= hi || (some && k > prefix)); };
    auto equal = [&](int i, uint32_t k) { return i >= lo && i < hi && some && k == prefix; };
    // A warp's rows by ballots, `at` the rows of each kind before them; put(place, row, e) for those that stay.
    uint2 at;
    const uint32_t below = (1u << lane) - 1;
    auto place = [&](int e, bool is_above, bool is_equal, auto put) {
        const uint32_t a = __ballot_sync(0xffffffffu, is_above), q = __ballot_sync(0xffffffffu, is_equal);
        if (q == 0) {
            if (is_above) put(at.x + __popc(a & below) + min(at.y, need), e);
        } else {
            const uint32_t y = at.y + __popc(q & below);
            if (is_above || (is_equal && y < need)) put(at.x + __popc(a & below) + min(y, need), e);
            at.y += __popc(q);
        }
        at.x += __popc(a);
    };
    // Kept rows of each kind in the warps before.
    auto before = [&](uint32_t x, uint32_t y) {
        x = __reduce_add_sync(0xffffffffu, x);
        y = __reduce_add_sync(0xffffffffu, y);
        if (lane == 0) warp_sums[warp] = make_uint2(x, y);
        __syncthreads();
        const uint2 o = lane < warp ? warp_sums[lane] : make_uint2(0, 0);
        return make_uint2(__reduce_add_sync(0xffffffffu, o.x), __reduce_add_sync(0xffffffffu, o.y));
    };
    if constexpr (RUN > 0) {
        uint32_t as = 0, es = 0;   // bit e: the thread's e-th row
#pragma unroll
        for (int e = 0; e < RUN; ++e) {
            const uint32_t k = sort_key(ws[e]);
            as |= (uint32_t)above(base + 32 * e, k) << e;
            es |= (uint32_t)equal(base + 32 * e, k) << e;
        }
        // The weights go along: they were read before the barrier and are stored after it, so in place too.
        at = before(__popc(as), __popc(es));
#pragma unroll
        for (int e = 0; e < RUN; ++e)
            place(e, as >> e & 1, es >> e & 1, [&](uint32_t p, int) {
                kept[p] = base + 32 * e;
                w_out[p] = ws[e];
            });
    } else {
        uint32_t x = 0, y = 0;
        each([&](int i, uint32_t k) {
            x += above(i, k);
            y += equal(i, k);
        });
        at = before(x, y);
        each([&](int i, uint32_t k) { place(i, above(i, k), equal(i, k), [&](uint32_t p, int row) { kept[p] = row; }); });
        __syncthreads();
        // The weights follow in tiles: in place, a tile's stores come after its loads.
        for (int i0 = 0; i0 < keep; i0 += SEL_THREADS) {
            const int i = i0 + t;
            const float x = i < keep ? w[kept[i]] : 0.f;
            if (w_out == w) __syncthreads();
            if (i < keep) w_out[i] = x;
        }
    }
}

struct GatherArgs {
    const uint8_t *k, *v;
    uint8_t *ok, *ov;
    long long cs, rs, hs, ls;        // strides in bytes
    long long ocs, ors, ohs, ols;
    int caches, K, keep, chunks;     // chunks: 16-byte chunks of a row
    const int* kept;
    const int* length;
    int* length_out;
    int rows;
    int in_place;
};

constexpr int GA_THREADS = 256;
constexpr int GA_UNROLL = 8;

// LANES: 16-byte chunks of a slice.
template <int LANES>
__global__ void __launch_bounds__(GA_THREADS) k_kv_gather(const __grid_constant__ GatherArgs a) {
    constexpr int ROWS = GA_THREADS / LANES;   // rows of one load
    const int item = blockIdx.y;   // (layer, cache, head)
    const int h = item % a.K, c = (item / a.K) % a.caches, l = item / (a.K * a.caches);
    const int slices = (a.chunks + LANES - 1) / LANES;
    const bool is_v = (int)blockIdx.x >= slices;
    const int ch = (blockIdx.x - (is_v ? slices : 0)) * LANES + (threadIdx.x & (LANES - 1));
    const int r0 = threadIdx.x / LANES;
    const uint8_t* src = (is_v ? a.v : a.k) + l * a.ls + c * a.cs + h * a.hs + ch * 16;
    uint8_t* dst = (is_v ? a.ov : a.ok) + l * a.ols + c * a.ocs + h * a.ohs + ch * 16;
    const int* kept = a.kept + (long long)item * a.keep;
    const bool mine = ch < a.chunks;
    ptx::grid_dep_wait();   // the choice
    for (int i0 = (int)blockIdx.z * ROWS * GA_UNROLL; i0 < a.keep; i0 += (int)gridDim.z * ROWS * GA_UNROLL) {
        uint4 x[GA_UNROLL];
        int r[GA_UNROLL];
#pragma unroll
        for (int u = 0; u < GA_UNROLL; ++u) {
            const int i = i0 + u * ROWS + r0;
            r[u] = i < a.keep && mine ? kept[i] : -1;
            if (a.in_place && r[u] == i) r[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < GA_UNROLL; ++u)
            if (r[u] >= 0) x[u] = *(const uint4*)(src + r[u] * a.rs);
        if (a.in_place) __syncthreads();
#pragma unroll
        for (int u = 0; u < GA_UNROLL; ++u)
            if (r[u] >= 0) *(uint4*)(dst + (long long)(i0 + u * ROWS + r0) * a.ors) = x[u];
    }
    // The choice has read the lengths: one thread of each cache's first block replaces its length.
    if (blockIdx.x == 0 && blockIdx.z == 0 && l == 0 && h == 0 && threadIdx.x == 0)
        a.length_out[c] = min(min(max(a.length[c], 0), a.rows), a.keep);
}

}  // namespace

jpi_status launch_kv_evict(const jpi_kv_handle* h, const jpi_kv_cache& src, const float* w, const int* length, int layers,
                           int caches, int keep, int sink, int recent, const jpi_kv_cache& dst, float* w_out,
                           int* length_out, int* kept, cudaStream_t st) {
    const int items = layers * caches * h->K;
    JPI_TRY(kv_start(src.rows <= SEL_THREADS ? k_kv_select<1>
                                             : src.rows <= 4 * SEL_THREADS ? k_kv_select<4>
                                                                           : src.rows <= 16 * SEL_THREADS ? k_kv_select<16> : k_kv_select<0>,
                     items, SEL_THREADS, 0, false, st, w, length, src.rows, caches, h->K, keep, sink, recent, dst.rows, w_out, kept));
    const long long e = h->bf16 ? 2 : 4;
    GatherArgs a = {};
    a.k = (const uint8_t*)src.k;
    a.v = (const uint8_t*)src.v;
    a.ok = (uint8_t*)dst.k;
    a.ov = (uint8_t*)dst.v;
    a.cs = src.cache_stride * e;
    a.rs = src.row_stride * e;
    a.hs = src.head_stride * e;
    a.ls = src.layer_stride * e;
    a.ocs = dst.cache_stride * e;
    a.ors = dst.row_stride * e;
    a.ohs = dst.head_stride * e;
    a.ols = dst.layer_stride * e;
    a.caches = caches;
    a.K = h->K;
    a.keep = keep;
    a.chunks = (int)(h->D * e / 16);
    a.kept = kept;
    a.length = length;
    a.length_out = length_out;
    a.rows = src.rows;
    a.in_place = src.k == dst.k;
    // Whole rows (to 512 bytes) where that still leaves two blocks an SM, else narrower slices: in place a slice's rows are
    // one block's.
    int lanes = 32;
    while (lanes > 1 && lanes / 2 >= a.chunks) lanes /= 2;
    auto blocks_of = [&](int n) { return 2ll * ((a.chunks + n - 1) / n) * items; };
    const int tile = GA_THREADS / lanes * GA_UNROLL;
    int gz = 1;
    if (a.in_place) {
        while (lanes > 2 && blocks_of(lanes) < 2ll * h->num_sms) lanes /= 2;
    } else {
        const int tiles = (keep + tile - 1) / tile;
        gz = (int)std::max(1ll, std::min({(long long)tiles, 8ll * h->num_sms / blocks_of(lanes), 65535ll}));
    }
    return kv_start(lanes == 32 ? k_kv_gather<32>
                                : lanes == 16 ? k_kv_gather<16>
                                              : lanes == 8 ? k_kv_gather<8> : lanes == 4 ? k_kv_gather<4> : lanes == 2 ? k_kv_gather<2> : k_kv_gather<1>,
                    dim3((unsigned)(blocks_of(lanes) / items), (unsigned)items, (unsigned)gz), GA_THREADS, 0, h->pdl, st, a);
}

}  // namespace jpi
