// What the kernels over windows share: which rows a tile of query rows sees, block by block of keys.
#pragma once

#include "kv_span.h"

namespace jpi {
namespace {

// First row of the window of a token that counts n rows.
__device__ __forceinline__ int span_first(const KvSpan& s, int n) { return max(n - s.window, 0); }
__device__ __forceinline__ bool span_sees(const KvSpan& s, int row, int n, int first) {
    return row < n && (row < s.sink || row >= first);
}

// The blocks of KEYS rows that a tile reads: those of the first `sink` rows, and those from the lowest first row of its windows to
// its largest count. The rows between are no block of the tile. (Where the counts lie far apart, rows that none of its tokens sees are
// among them: a test of every block against every count would cost the calls whose tokens follow one another, which is nearly all.)
template <int KEYS>
struct SpanBlocks {
    int head, skip, count;   // blocks of the first rows, blocks left out behind them, blocks in all
    // n: the largest count of the tile's rows; first: the lowest first row of those with a count.
    __device__ __forceinline__ SpanBlocks(const KvSpan& s, int n, int first) {
        const int end = (n + KEYS - 1) / KEYS;
        head = (min(s.sink, n) + KEYS - 1) / KEYS;
        skip = max(min(first, n) / KEYS - head, 0);
        count = end - skip;
    }
    __device__ __forceinline__ int row(int block) const { return (block < head ? block : block + skip) * KEYS; }
};

}  // namespace
}  // namespace jpi
