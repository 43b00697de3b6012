// KV-cache operators (include/jpi_kv.h): the handle and the launchers of its kernels.
#pragma once
#include "../jpi_internal.h"
#include "jpi_kv.h"

struct jpi_kv_handle {
    jpi_kv_config cfg;
    int device = 0;
    int num_sms = 0;
    bool bf16 = true;
    int H, K, D, gq;          // query heads, KV heads, head dim, H / K
    float scale;              // of the scores
    bool rope = false;
    jpi_kv_rope rope_cfg = {};
    uint64_t* turns = nullptr;   // [dim / 2] turns per position of each rotary pair, in units of 2^-64
    void* ws = nullptr;          // partial outputs and statistics of jpi_kv_attend
    size_t ws_bytes = 0;
    int* dev_err = nullptr;
    bool pdl = true;             // kernels of one call may start before the one before them has finished
    int tiles = -1;              // attend, weigh: the tensor-core tiles never, (1) wherever they fit, (-1) by size
    size_t device_bytes = 0;
    std::vector<void*> allocations;
};

namespace jpi {

// n / d for 0 <= n < 2^31 by a multiplication: with 2^s >= d > 2^(s-1) and m = floor(2^32 (2^s - d) / d) + 1,
// n / d = (floor(m n / 2^32) + n) >> s.
struct KvDiv {
    uint32_t d = 1, m = 1, s = 0;
    KvDiv() = default;
    explicit KvDiv(uint32_t div) : d(div) {
        while ((1ull << s) < div) ++s;
        m = (uint32_t)(((1ull << 32) * ((1ull << s) - div)) / div + 1);
    }
#ifdef __CUDACC__
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, m) + n) >> s; }
    __device__ __forceinline__ uint32_t div(uint32_t n, uint32_t& rem) const {
        const uint32_t q = div(n);
        rem = n - q * d;
        return q;
    }
#endif
};

// One side of a call's keys as the kernels read them: `n` caches of at most `rows` rows.
struct KvSide {
    const void *k = nullptr, *v = nullptr;
    long long cs = 0, rs = 0, hs = 0;   // cache, row and head strides (elements)
    int rows = 0;
    const int* len = nullptr;           // [groups] lengths (prefix) or [batch][tokens] seen counts (own)
};

// Arguments of attend and weigh, shared by their kernels.
struct KvCall {
    const void* q = nullptr;
    long long q_stride = 0;
    int batch = 0, tokens = 0, groups = 1;
    int H = 0, K = 0, D = 0, gq = 0;
    float scale = 0.f;                  // of the scores
    KvSide prefix, own;                 // rows == 0: absent
    KvDiv by_gq, by_K;
};

// Bytes of workspace that any attend within the maxima needs (kv_attend.cu).
size_t kv_attend_ws_bytes(const jpi_kv_handle* h);
jpi_status kv_attend_prepare(jpi_kv_handle* h);

jpi_status kv_append_prepare();
jpi_status launch_kv_append(const jpi_kv_handle* h, const void* q, long long q_stride, const void* k, long long k_stride,
                            const void* v, long long v_stride, const int* position, const int* row, int batch,
                            int tokens, void* q_out, const jpi_kv_cache* cache, cudaStream_t st);
jpi_status launch_kv_attend(jpi_kv_handle* h, const KvCall& c, void* out, float* lse, cudaStream_t st);
jpi_status launch_kv_weigh(jpi_kv_handle* h, const KvCall& c, const float* lse, float decay, const float* prefix_in,
                           float* prefix_out, const float* own_in, float* own_out, cudaStream_t st);
jpi_status launch_kv_evict(const jpi_kv_handle* h, const jpi_kv_cache& src, const float* w, const int* length, int layers,
                           int caches, int keep, int sink, int recent, const jpi_kv_cache& dst, float* w_out,
                           int* length_out, int* kept, cudaStream_t st);

// An ordinary launch, or with `early` one that starts while the kernel before it runs; in clusters of `ranks` blocks.
template <typename... Params, typename... Args>
jpi_status kv_start_clusters(void (*kernel)(Params...), dim3 grid, unsigned ranks, int threads, size_t smem, bool early,
                             cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    cfg.attrs = at;
    if (early) {
        at[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (ranks > 1) {
        at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        at[cfg.numAttrs].val.clusterDim.x = ranks;
        at[cfg.numAttrs].val.clusterDim.y = 1;
        at[cfg.numAttrs++].val.clusterDim.z = 1;
    }
    JPI_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    return JPI_OK;
}
template <typename... Params, typename... Args>
jpi_status kv_start(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, bool early, cudaStream_t st,
                    const Args&... args) {
    return kv_start_clusters(kernel, grid, 1, threads, smem, early, st, args...);
}

}  // namespace jpi
