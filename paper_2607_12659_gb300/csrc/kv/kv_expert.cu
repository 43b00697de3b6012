// The expert's use of the KV-cache operators (kv_expert.h).
//
// The store [L][maxB][kv_rows][D] is, layer by layer, `cur_batch` prefixes in rows 0 .. P - 1 of the first
// slots and the suffix keys of every request in rows P .. of its own slot: two of jpi_kv.h's caches at the same strides.
// Row b S + i of the queries, S suffix tokens a request, sees the whole prefix and its request's first `seen` suffix
// rows: the state and context tokens each other, the actions all.

#include "kv_expert.h"

namespace jpi {
namespace {

__global__ void k_fill_seen(int* seen, int* len, int B, int S, int nctx, int G, int P) {
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < B * S; i += gridDim.x * blockDim.x) {
        seen[i] = i % S < nctx ? nctx : S;
        if (i < G) len[i] = P;   // (G <= B * S)
    }
}
__global__ void k_fill_len(int* len, int n, int P) {
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) len[i] = P;
}
// As the expert's own table is made: the angle in 64 bits, its cosine and sine rounded.
__global__ void k_fill_rope(float2* rope, const int* start, int S, int half, double base) {
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < S * half; i += gridDim.x * blockDim.x) {
        const int d = i % half;
        double s, c;
        sincos((double)(*start + i / half) * pow(base, -1.0 * d / half), &s, &c);
        rope[i] = make_float2((float)c, (float)s);
    }
}
// Appended tokens [B][T]: positions p0 + t, rows r0 + t; the suffix follows at p0 + T.
__global__ void k_fill_tokens(int* position, int* row, int* start, int n, int T, int p0, int r0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *start = p0 + T;
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) {
        position[i] = p0 + i % T;
        row[i] = r0 + i % T;
    }
}
int grid_of(long long n) { return (int)(n < 256 * 256 ? (n + 255) / 256 : 256); }

size_t elem(const jpi_handle* h) { return h->bf16 ? 2 : 4; }

// Rows of layer l's store from `row0` on, as caches.
jpi_kv_cache store_of(const jpi_handle* h, int l, int row0, int rows) {
    jpi_kv_cache c = {};
    const size_t at = ((size_t)l * h->maxB * h->kv_rows + row0) * h->D * elem(h);
    c.k = static_cast<char*>(h->kv_k) + at;
    c.v = static_cast<char*>(h->kv_v) + at;
    c.cache_stride = (long long)h->kv_rows * h->D;
    c.row_stride = c.head_stride = h->D;
    c.layer_stride = (long long)h->maxB * h->kv_rows * h->D;
    c.rows = rows;
    return c;
}
KvSide side_of(const jpi_kv_cache& c, const int* len) {
    KvSide s;
    s.k = c.k;
    s.v = c.v;
    s.cs = c.cache_stride;
    s.rs = c.row_stride;
    s.hs = c.head_stride;
    s.rows = c.rows;
    s.len = len;
    return s;
}

}  // namespace

jpi_status expert_kv_create(jpi_handle* h, ExpertKv* e) {
    jpi_kv_config cfg = {};
    cfg.n_heads = h->H;
    cfg.n_kv_heads = 1;
    cfg.head_dim = h->D;
    cfg.max_batch = h->maxB;
    cfg.max_tokens = h->maxS;
    cfg.precision = h->bf16 ? JPI_BF16 : JPI_FP32;
    jpi_kv_rope rope = {};
    rope.dim = h->D;
    rope.layout = JPI_ROPE_HALF;
    rope.base = h->cfg.rope_base;
    rope.mscale = 1.f;
    JPI_TRY(jpi_kv_create(&cfg, h->cfg.rope_base >= 1.f ? &rope : nullptr, &e->kv));
    e->kv->pdl = h->pdl;
    e->kv->dev_err = h->dev_err;   // what its kernels report is the expert's status
    const size_t ints = (size_t)h->maxB * h->maxS + h->maxB + 2 * (size_t)h->maxB * h->maxP + (size_t)h->L * h->maxB * h->maxP + 1;
    const size_t bytes = (size_t)h->maxS * (h->D / 2) * sizeof(float2) + ints * sizeof(int) + (size_t)h->maxMt * h->H * sizeof(float);
    void* p = nullptr;
    if (cudaMalloc(&p, bytes) != cudaSuccess) {
        cudaGetLastError();
        expert_kv_destroy(e);
        set_error("cudaMalloc of %zu bytes failed", bytes);
        return JPI_ERR_OOM;
    }
    h->allocations.push_back(p);
    h->device_bytes += bytes + e->kv->device_bytes;
    e->rope = static_cast<float2*>(p);
    e->lse = reinterpret_cast<float*>(e->rope + (size_t)h->maxS * (h->D / 2));
    e->seen = reinterpret_cast<int*>(e->lse + (size_t)h->maxMt * h->H);
    e->len = e->seen + (size_t)h->maxB * h->maxS;
    e->position = e->len + h->maxB;
    e->row = e->position + (size_t)h->maxB * h->maxP;
    e->kept = e->row + (size_t)h->maxB * h->maxP;
    e->start = e->kept + (size_t)h->L * h->maxB * h->maxP;
    return JPI_OK;
}

void expert_kv_destroy(ExpertKv* e) {
    jpi_kv_destroy(e->kv);
    e->kv = nullptr;
}

jpi_status expert_kv_fill(jpi_handle* h, const ExpertKv& e, int B, int C, int share, cudaStream_t st) {
    const int S = C + h->n_ctx();
    k_fill_seen<<<grid_of((long long)B * S), 256, 0, st>>>(e.seen, e.len, B, S, h->n_ctx(), B / share, h->cur_prefix);
    JPI_CUDA_TRY(cudaGetLastError());
    return JPI_OK;
}

jpi_status expert_kv_attention(jpi_handle* h, const ExpertKv& e, int l, int B, int C, int share, float* w, float decay,
                               cudaStream_t st) {
    KvCall c;
    c.q = h->q;
    c.q_stride = (long long)h->H * h->D;
    c.batch = B;
    c.tokens = C + h->n_ctx();
    c.groups = B / share;
    c.H = h->H;
    c.K = 1;
    c.D = h->D;
    c.gq = h->H;
    c.scale = e.kv->scale;
    c.by_gq = KvDiv((uint32_t)h->H);
    c.by_K = KvDiv(1u);
    c.prefix = side_of(store_of(h, l, 0, h->cur_prefix), e.len);
    c.own = side_of(store_of(h, l, h->cur_prefix, c.tokens), e.seen);
    JPI_TRY(launch_kv_attend(e.kv, c, h->o, w ? e.lse : nullptr, st));
    if (!w) return JPI_OK;
    c.own = KvSide();
    return launch_kv_weigh(e.kv, c, e.lse, decay, w, w, nullptr, nullptr, st);
}

jpi_status expert_kv_evict(jpi_handle* h, const ExpertKv& e, float* w, int keep, int sink, int recent, int* kept, cudaStream_t st) {
    k_fill_len<<<grid_of(h->cur_batch), 256, 0, st>>>(e.len, h->cur_batch, h->cur_prefix);
    JPI_CUDA_TRY(cudaGetLastError());
    const jpi_kv_cache c = store_of(h, 0, 0, h->cur_prefix);
    return launch_kv_evict(e.kv, c, w, e.len, h->L, h->cur_batch, keep, sink, recent, c, w, e.len, kept ? kept : e.kept, st);
}

jpi_status expert_kv_rope(jpi_handle* h, const ExpertKv& e, int C, cudaStream_t st) {
    const int S = C + h->n_ctx();
    k_fill_rope<<<grid_of((long long)S * (h->D / 2)), 256, 0, st>>>(e.rope, e.start, S, h->D / 2, h->cfg.rope_base);
    JPI_CUDA_TRY(cudaGetLastError());
    return JPI_OK;
}

jpi_status expert_kv_append(jpi_handle* h, const ExpertKv& e, const void* const* k_layers, const void* const* v_layers, int tokens,
                            int position, cudaStream_t st) {
    const int n = h->cur_batch * tokens;
    k_fill_tokens<<<grid_of(n), 256, 0, st>>>(e.position, e.row, e.start, n, tokens, position, h->cur_prefix);
    JPI_CUDA_TRY(cudaGetLastError());
    for (int l = 0; l < h->L; ++l) {
        const jpi_kv_cache c = store_of(h, l, 0, h->kv_rows);
        JPI_TRY(launch_kv_append(e.kv, nullptr, 0, k_layers[l], h->D, v_layers[l], h->D, e.position, e.row, h->cur_batch, tokens,
                                 nullptr, &c, st));
    }
    return JPI_OK;
}

}  // namespace jpi
