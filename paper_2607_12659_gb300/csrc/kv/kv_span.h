// Attention over windows of a cache, in the handle's type or in 8 bits (jpi_kv_attend_window, jpi_kv8_attend): kv_span.cu.
#pragma once
#include "kv.h"

namespace jpi {

// What a query token sees of the rows before its count n, and how the cache is held: rows r < n with r < sink or r >= n - window.
// The cache itself is the call's `own` side; codes of 8 bits have one byte an element, so that strides are bytes there.
struct KvSpan {
    int window = 0x7fffffff, sink = 0;
    const uint8_t *ks = nullptr, *vs = nullptr;   // scales [caches][K][nblk], or NULL: not in 8 bits
    int n_log2 = 0, nblk = 0;                     // rows of a block (log2), blocks of a cache
};

jpi_status launch_kv_span(jpi_kv_handle* h, const KvCall& c, const KvSpan& s, void* out, float* lse, cudaStream_t st);

// On tensor-core tiles of 128 query rows (kv_span_t5.cu): the key splits, of at most `room`, that a call takes there; 0: it does not.
// `joined`: the launch joins them itself.
jpi_status kv_span_tiles_prepare(jpi_kv_handle* h);
int kv_span_tiles_plan(const jpi_kv_handle* h, const KvCall& c, const KvSpan& s, long long room, bool* joined);
// Its parts in `po` [splits][rows][D] and `pml` [rows][splits], or of one, or joined, the result itself.
jpi_status launch_kv_span_tiles(jpi_kv_handle* h, const KvCall& c, const KvSpan& s, int splits, bool joined, float* po, float2* pml, void* out,
                                float* lse, cudaStream_t st);

}  // namespace jpi
