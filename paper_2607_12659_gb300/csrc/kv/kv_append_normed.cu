// Norms of queries and keys for each head, rotary coding and cache write in one pass (jpi_kv_append_normed).
//
//   y = rope(x / sqrt(mean(x^2) + eps) * w)
//
// Bound by memory: every element is read and written once. Warps stay and take tokens in turn, whose heads are
// held by groups of lanes (kv_heads.cuh).

#include "kv_heads.cuh"

namespace jpi {
namespace {

struct NormedArgs {
    HeadArgs h;
    CodeTokens ct;
    const int* row;
    void *ck, *cv;
    long long cs, rs, hs;
    int rows;
};

constexpr int AN_THREADS = 128, AN_BLOCKS = 7;   // of a block; blocks of an SM

template <typename E, int MODE>
__global__ void __launch_bounds__(AN_THREADS, AN_BLOCKS) k_kv_append_normed(const __grid_constant__ NormedArgs a) {
    __shared__ CodeWeights weights;
    __shared__ __align__(16) CodeTable table[AN_THREADS / 32];
    auto place = [&](int tok) {
        const int r = a.row[tok];
        return r < a.rows ? r : -1;
    };
    auto at = [&](long long tok, int row) { return (long long)a.h.by_tokens.div((uint32_t)tok) * a.cs + row * a.rs; };
    load_weights<E, MODE>(a.h, weights);
    __syncthreads();
    code_tokens<E, MODE>(a.h, a.ct, weights, table[threadIdx.x >> 5], blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5),
                         gridDim.x * (blockDim.x >> 5), static_cast<E*>(a.ck), static_cast<E*>(a.cv), a.hs, place, at);
}

template <typename E>
jpi_status launch(const jpi_kv_handle* h, const NormedArgs& a, int mode, cudaStream_t st) {
    auto* const kernel = mode == RM_NONE ? k_kv_append_normed<E, RM_NONE>
                                         : mode == RM_HALF ? k_kv_append_normed<E, RM_HALF>
                                                           : mode == RM_INTER ? k_kv_append_normed<E, RM_INTER> : k_kv_append_normed<E, RM_SCALAR>;
    return kv_start(kernel, dim3(code_blocks(h, a.ct, AN_THREADS, AN_BLOCKS)), AN_THREADS, 0, false, st, a);
}

}  // namespace

jpi_status launch_kv_append_normed(const jpi_kv_handle* h, const void* q, long long q_stride, const void* k, long long k_stride,
                                   const void* v, long long v_stride, const jpi_kv_norm* norm, const int* position, const int* row,
                                   int batch, int tokens, void* q_out, const jpi_kv_cache* cache, cudaStream_t st) {
    NormedArgs a = {};
    a.h.q = q;
    a.h.k = k;
    a.h.v = v;
    a.h.q_stride = q_stride;
    a.h.k_stride = k_stride;
    a.h.v_stride = v_stride;
    a.h.position = position;
    a.h.q_out = q_out;
    a.h.H = q ? h->H : 0;
    a.h.K = k ? h->K : 0;
    a.h.batch = batch;
    a.h.tokens = tokens;
    a.h.norm = true;
    a.h.q_weight = norm->q_weight;
    a.h.k_weight = norm->k_weight;
    a.h.eps = norm->eps;
    a.row = row;
    a.rows = 0x7fffffff;
    if (cache) {
        a.ck = cache->k;
        a.cv = cache->v;
        a.cs = cache->cache_stride;
        a.rs = cache->row_stride;
        a.hs = cache->head_stride;
        a.rows = cache->rows;
    }
    const int mode = plan_code_tokens(h, a.h, a.ct, v ? h->K : 0);
    return h->bf16 ? launch<__nv_bfloat16>(h, a, mode, st) : launch<float>(h, a, mode, st);
}

}  // namespace jpi
