// C-ABI entry points of the KV-cache operators (include/jpi_kv.h): argument checks, the handle and
// its rotary table. The kernels are in kv_append.cu, kv_attend.cu, kv_weigh.cu and kv_evict.cu.

#include "kv.h"
#include "kv_weigh.h"

#include <cstdlib>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

namespace jpi {
namespace {

jpi_status fail(jpi_status s, const char* fmt, ...) {
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    set_error("%s", msg);
    return s;
}

jpi_status kv_alloc(jpi_kv_handle* h, void** p, size_t bytes) {
    h->allocations.reserve(h->allocations.size() + 1);   // (may throw, so before there is something to lose)
    cudaError_t e = cudaMalloc(p, bytes ? bytes : 16);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(JPI_ERR_OOM, "cudaMalloc(%zu bytes) failed: %s", bytes, cudaGetErrorString(e));
    }
    h->allocations.push_back(*p);
    h->device_bytes += bytes;
    return JPI_OK;
}

void free_kv(jpi_kv_handle* h) {
    if (!h) return;
    int cur = 0;
    const bool back = cudaGetDevice(&cur) == cudaSuccess && cur != h->device;
    cudaSetDevice(h->device);
    cudaDeviceSynchronize();
    for (void* p : h->allocations) cudaFree(p);
    if (back) cudaSetDevice(cur);
    cudaGetLastError();
    delete h;
}

jpi_status check_rope(const jpi_kv_rope* r, int D) {
    if (r->dim < 2 || r->dim % 2 || r->dim > D)
        return fail(JPI_ERR_INVALID_ARG, "rope dim %d must be even and in 2..%d", r->dim, D);
    if (r->layout != JPI_ROPE_HALF && r->layout != JPI_ROPE_INTERLEAVED)
        return fail(JPI_ERR_INVALID_ARG, "unknown rope layout %d", r->layout);
    if (r->scaling < JPI_ROPE_PLAIN || r->scaling > JPI_ROPE_BY_PARTS)
        return fail(JPI_ERR_INVALID_ARG, "unknown rope scaling %d", r->scaling);
    if (!(r->base >= 1.f) || std::isinf(r->base) || !(r->mscale > 0.f) || std::isinf(r->mscale))
        return fail(JPI_ERR_INVALID_ARG, "rope base must be >= 1 and mscale > 0, both finite");
    if (r->scaling != JPI_ROPE_PLAIN && (!(r->factor >= 1.f) || std::isinf(r->factor)))
        return fail(JPI_ERR_INVALID_ARG, "rope factor must be >= 1 and finite");
    if (r->scaling == JPI_ROPE_NTK && r->dim < 4)
        return fail(JPI_ERR_INVALID_ARG, "JPI_ROPE_NTK needs a rope dim of at least 4");
    if (r->scaling == JPI_ROPE_BY_PARTS && (!(r->low < r->high) || std::isinf(r->low) || std::isinf(r->high) || r->original < 1))
        return fail(JPI_ERR_INVALID_ARG, "JPI_ROPE_BY_PARTS needs low < high and original >= 1");
    return JPI_OK;
}

// Turns per position of pair i (angle / 2 pi, at most 1 / 2 pi), in 64 bits.
double turns_of(const jpi_kv_rope& r, int i) {
    double base = r.base;
    if (r.scaling == JPI_ROPE_NTK) base *= std::pow((double)r.factor, (double)r.dim / (r.dim - 2));
    double th = std::pow(base, -2.0 * i / r.dim);
    if (r.scaling == JPI_ROPE_LINEAR) th /= r.factor;
    constexpr double TWO_PI = 6.283185307179586476925;
    if (r.scaling == JPI_ROPE_BY_PARTS) {
        const double rot = r.original * th / TWO_PI;
        const double g = std::fmin(1.0, std::fmax(0.0, (rot - r.low) / ((double)r.high - r.low)));
        th = (1.0 - g) * th / r.factor + g * th;
    }
    return th / TWO_PI;
}

jpi_status check_handle(const jpi_kv_handle* h) {
    if (!h) return fail(JPI_ERR_INVALID_ARG, "handle is NULL");
    int dev = -1;
    JPI_CUDA_TRY(cudaGetDevice(&dev));
    if (dev != h->device)
        return fail(JPI_ERR_INVALID_ARG, "the current device is %d, the handle's %d", dev, h->device);
    return JPI_OK;
}

size_t elem(const jpi_kv_handle* h) { return h->bf16 ? 2 : 4; }
bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

jpi_status check_count(const jpi_kv_handle* h, int batch, int tokens) {
    if (batch < 1 || tokens < 1) return fail(JPI_ERR_INVALID_ARG, "batch and tokens must be >= 1");
    if (batch > h->cfg.max_batch || tokens > h->cfg.max_tokens)
        return fail(JPI_ERR_SHAPE, "batch %d / tokens %d exceed the maxima %d / %d", batch, tokens, h->cfg.max_batch,
                    h->cfg.max_tokens);
    return JPI_OK;
}

// A token stride of `heads` heads.
jpi_status check_stride(const jpi_kv_handle* h, const char* what, const void* p, long long stride, int heads) {
    if (!aligned(p)) return fail(JPI_ERR_INVALID_ARG, "%s is not 16-byte aligned", what);
    if (stride < (long long)heads * h->D || stride > (1ll << 40) || (stride * (long long)elem(h)) % 16)
        return fail(JPI_ERR_INVALID_ARG, "%s stride %lld must cover a token and be a multiple of 16 bytes", what, stride);
    return JPI_OK;
}

jpi_status check_cache(const jpi_kv_handle* h, const char* what, const jpi_kv_cache* c, int n, int layers, bool need_v) {
    if (!c->k || (need_v && !c->v)) return fail(JPI_ERR_INVALID_ARG, "%s: k or v is NULL", what);
    if (!aligned(c->k) || (c->v && !aligned(c->v))) return fail(JPI_ERR_INVALID_ARG, "%s: k or v is not 16-byte aligned", what);
    if (c->rows < 1 || c->rows > (1 << 30)) return fail(JPI_ERR_INVALID_ARG, "%s: rows %d must be in 1..2^30", what, c->rows);
    const struct { const char* name; long long stride, size; } s[4] = {{"cache_stride", c->cache_stride, n},
        {"row_stride", c->row_stride, c->rows}, {"head_stride", c->head_stride, h->K}, {"layer_stride", c->layer_stride, layers}};
    for (const auto& d : s)
        if (d.size > 1 && (d.stride < h->D || d.stride > (1ll << 60) / d.size || (d.stride * (long long)elem(h)) % 16))
            return fail(JPI_ERR_INVALID_ARG, "%s: %s %lld must be at least head_dim and a multiple of 16 bytes", what, d.name,
                        d.stride);
    return JPI_OK;
}

KvSide side_of(const jpi_kv_cache* c, const int* len) {
    KvSide s;
    if (!c) return s;
    s.k = c->k;
    s.v = c->v;
    s.cs = c->cache_stride;
    s.rs = c->row_stride;
    s.hs = c->head_stride;
    s.rows = c->rows;
    s.len = len;
    return s;
}

// The arguments that attend and weigh share.
jpi_status make_call(const jpi_kv_handle* h, const void* q, long long q_stride, int batch, int tokens,
                     const jpi_kv_cache* prefix, int groups, const int* prefix_len, const jpi_kv_cache* own,
                     const int* seen, bool need_v, KvCall* c) {
    JPI_TRY(check_handle(h));
    JPI_TRY(check_count(h, batch, tokens));
    if (!q) return fail(JPI_ERR_INVALID_ARG, "q is NULL");
    if (!prefix && !own) return fail(JPI_ERR_INVALID_ARG, "prefix and own are both NULL");
    if ((prefix != nullptr) != (prefix_len != nullptr) || (own != nullptr) != (seen != nullptr))
        return fail(JPI_ERR_INVALID_ARG, "prefix goes with prefix_len, own with seen");
    if (groups < 1 || batch % groups) return fail(JPI_ERR_INVALID_ARG, "groups %d must divide the batch %d", groups, batch);
    if (!prefix && groups != 1) return fail(JPI_ERR_INVALID_ARG, "groups is 1 without a prefix");
    JPI_TRY(check_stride(h, "q", q, q_stride, h->H));
    if (prefix) JPI_TRY(check_cache(h, "prefix", prefix, groups, 1, need_v));
    if (own) JPI_TRY(check_cache(h, "own", own, batch, 1, need_v));
    c->q = q;
    c->q_stride = q_stride;
    c->batch = batch;
    c->tokens = tokens;
    c->groups = groups;
    c->H = h->H;
    c->K = h->K;
    c->D = h->D;
    c->gq = h->gq;
    c->scale = h->scale;
    c->by_gq = KvDiv((uint32_t)h->gq);
    c->by_K = KvDiv((uint32_t)h->K);
    c->prefix = side_of(prefix, prefix_len);
    c->own = side_of(own, seen);
    return JPI_OK;
}

}  // namespace
}  // namespace jpi

using namespace jpi;

extern "C" {

JPI_API jpi_status jpi_kv_create(const jpi_kv_config* cfg, const jpi_kv_rope* rope, jpi_kv_handle** out) {
    clear_error();
    if (!out) return fail(JPI_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    if (!cfg) return fail(JPI_ERR_INVALID_ARG, "config is NULL");
    if (cfg->precision != JPI_BF16 && cfg->precision != JPI_FP32)
        return fail(JPI_ERR_INVALID_ARG, "unknown precision %d", (int)cfg->precision);
    const int mult = cfg->precision == JPI_BF16 ? 8 : 4;
    if (cfg->n_heads < 1 || cfg->n_kv_heads < 1 || cfg->n_heads % cfg->n_kv_heads)
        return fail(JPI_ERR_INVALID_ARG, "n_heads %d must be a multiple of n_kv_heads %d", cfg->n_heads, cfg->n_kv_heads);
    if (cfg->n_heads > 1024) return fail(JPI_ERR_UNSUPPORTED, "n_heads must be at most 1024");
    if (cfg->head_dim < mult || cfg->head_dim > 256 || cfg->head_dim % mult)
        return fail(JPI_ERR_UNSUPPORTED, "head_dim %d must be a multiple of %d and at most 256", cfg->head_dim, mult);
    if (cfg->max_batch < 1 || cfg->max_tokens < 1) return fail(JPI_ERR_INVALID_ARG, "max_batch and max_tokens must be >= 1");
    if (cfg->max_batch > 65535 || (long long)cfg->max_batch * cfg->max_tokens * cfg->n_heads > (1ll << 28))
        return fail(JPI_ERR_SHAPE, "maxima too large");
    if (cfg->scale != 0.f && !(cfg->scale >= 0x1p-32f && cfg->scale <= 0x1p32f))
        return fail(JPI_ERR_INVALID_ARG, "scale must be 0 or in 2^-32 .. 2^32");
    if (rope) JPI_TRY(check_rope(rope, cfg->head_dim));
    jpi_kv_handle* h = new (std::nothrow) jpi_kv_handle();
    if (!h) return fail(JPI_ERR_OOM, "host allocation failed");
    h->cfg = *cfg;
    h->bf16 = cfg->precision == JPI_BF16;
    h->H = cfg->n_heads;
    h->K = cfg->n_kv_heads;
    h->D = cfg->head_dim;
    h->gq = h->H / h->K;
    // JPI_KV_TILES=0 / 1 fixes which kernels take the sides that both could.
    const char* tiles_env = std::getenv("JPI_KV_TILES");
    if (tiles_env && (tiles_env[0] == '0' || tiles_env[0] == '1')) h->tiles = tiles_env[0] - '0';
    h->scale = cfg->scale > 0.f ? cfg->scale : 1.f / sqrtf((float)h->D);
    auto setup = [&]() -> jpi_status {
        JPI_CUDA_TRY(cudaGetDevice(&h->device));
        JPI_CUDA_TRY(cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, h->device));
        JPI_TRY(kv_alloc(h, reinterpret_cast<void**>(&h->dev_err), sizeof(int)));
        JPI_CUDA_TRY(cudaMemset(h->dev_err, 0, sizeof(int)));
        if (rope) {
            h->rope = true;
            h->rope_cfg = *rope;
            std::vector<uint64_t> t((size_t)rope->dim / 2);
            for (size_t i = 0; i < t.size(); ++i) t[i] = (uint64_t)std::ldexp(turns_of(*rope, (int)i), 64);
            JPI_TRY(kv_alloc(h, reinterpret_cast<void**>(&h->turns), t.size() * sizeof(uint64_t)));
            JPI_CUDA_TRY(cudaMemcpy(h->turns, t.data(), t.size() * sizeof(uint64_t), cudaMemcpyHostToDevice));
        }
        h->ws_bytes = kv_attend_ws_bytes(h);
        JPI_TRY(kv_alloc(h, &h->ws, h->ws_bytes));
        JPI_TRY(kv_append_prepare());
        JPI_TRY(kv_weigh_prepare(h));
        return kv_attend_prepare(h);
    };
    jpi_status s;
    try {
        s = setup();
    } catch (const std::bad_alloc&) {
        s = fail(JPI_ERR_OOM, "host allocation failed");
    }
    if (s != JPI_OK) {
        free_kv(h);
        return s;
    }
    *out = h;
    return JPI_OK;
}

JPI_API jpi_status jpi_kv_destroy(jpi_kv_handle* h) {
    clear_error();
    free_kv(h);
    return JPI_OK;
}

JPI_API jpi_status jpi_kv_append(jpi_kv_handle* h, const void* q, long long q_stride, const void* k, long long k_stride,
                                 const void* v, long long v_stride, const int* position, const int* row, int batch,
                                 int tokens, void* q_out, const jpi_kv_cache* cache, void* stream) {
    clear_error();
    JPI_TRY(check_handle(h));
    JPI_TRY(check_count(h, batch, tokens));
    if (!q && !k) return fail(JPI_ERR_INVALID_ARG, "q and k are both NULL");
    if ((q != nullptr) != (q_out != nullptr)) return fail(JPI_ERR_INVALID_ARG, "q goes with q_out");
    if ((k != nullptr) != (cache != nullptr)) return fail(JPI_ERR_INVALID_ARG, "k goes with cache");
    if (v && !k) return fail(JPI_ERR_INVALID_ARG, "v without k");
    if (!position || !row) return fail(JPI_ERR_INVALID_ARG, "position or row is NULL");
    if (q) {
        JPI_TRY(check_stride(h, "q", q, q_stride, h->H));
        if (!aligned(q_out)) return fail(JPI_ERR_INVALID_ARG, "q_out is not 16-byte aligned");
    }
    if (k) {
        JPI_TRY(check_stride(h, "k", k, k_stride, h->K));
        if (v) JPI_TRY(check_stride(h, "v", v, v_stride, h->K));
        JPI_TRY(check_cache(h, "cache", cache, batch, 1, v != nullptr));
    }
    return launch_kv_append(h, q, q_stride, k, k_stride, v, v_stride, position, row, batch, tokens, q_out, cache,
                            (cudaStream_t)stream);
}

JPI_API jpi_status jpi_kv_attend(jpi_kv_handle* h, const void* q, long long q_stride, int batch, int tokens,
                                 const jpi_kv_cache* prefix, int groups, const int* prefix_len, const jpi_kv_cache* own,
                                 const int* seen, void* out, float* lse, void* stream) {
    clear_error();
    KvCall c;
    JPI_TRY(make_call(h, q, q_stride, batch, tokens, prefix, groups, prefix_len, own, seen, true, &c));
    if (!out || !aligned(out)) return fail(JPI_ERR_INVALID_ARG, "out is NULL or not 16-byte aligned");
    return launch_kv_attend(h, c, out, lse, (cudaStream_t)stream);
}

JPI_API jpi_status jpi_kv_weigh(jpi_kv_handle* h, const void* q, long long q_stride, const float* lse, int batch,
                                int tokens, const jpi_kv_cache* prefix, int groups, const int* prefix_len,
                                const jpi_kv_cache* own, const int* seen, float decay, const float* prefix_in,
                                float* prefix_out, const float* own_in, float* own_out, void* stream) {
    clear_error();
    KvCall c;
    JPI_TRY(make_call(h, q, q_stride, batch, tokens, prefix, groups, prefix_len, own, seen, false, &c));
    if (!lse) return fail(JPI_ERR_INVALID_ARG, "lse is NULL");
    if ((prefix != nullptr) != (prefix_out != nullptr) || (own != nullptr) != (own_out != nullptr))
        return fail(JPI_ERR_INVALID_ARG, "prefix goes with prefix_out, own with own_out");
    if ((prefix_in && !prefix_out) || (own_in && !own_out)) return fail(JPI_ERR_INVALID_ARG, "weights in without weights out");
    if (!(decay >= 0.f) || std::isinf(decay)) return fail(JPI_ERR_INVALID_ARG, "decay must be >= 0 and finite");
    return launch_kv_weigh(h, c, lse, decay, prefix_in, prefix_out, own_in, own_out, (cudaStream_t)stream);
}

JPI_API jpi_status jpi_kv_evict(jpi_kv_handle* h, const jpi_kv_cache* src, const float* w, const int* length, int layers,
                                int caches, int keep, int sink, int recent, const jpi_kv_cache* dst, float* w_out,
                                int* length_out, int* kept, void* stream) {
    clear_error();
    JPI_TRY(check_handle(h));
    if (!src || !dst || !w || !w_out || !length || !length_out || !kept) return fail(JPI_ERR_INVALID_ARG, "NULL argument");
    if (layers < 1 || caches < 1) return fail(JPI_ERR_INVALID_ARG, "layers and caches must be >= 1");
    if (layers > 65535 || caches > 65535 || (long long)layers * caches * h->K > 65535)
        return fail(JPI_ERR_SHAPE, "layers * caches * n_kv_heads must be at most 65535");
    JPI_TRY(check_cache(h, "src", src, caches, layers, true));
    JPI_TRY(check_cache(h, "dst", dst, caches, layers, true));
    if (keep < 1 || sink < 0 || recent < 0 || (long long)sink + recent > keep)
        return fail(JPI_ERR_INVALID_ARG, "keep %d must be >= 1 and hold sink %d and recent %d", keep, sink, recent);
    if (keep > src->rows || keep > dst->rows)
        return fail(JPI_ERR_SHAPE, "keep %d exceeds the caches' rows %d / %d", keep, src->rows, dst->rows);
    // In place, or apart: anything between would overwrite rows that are still to be read.
    auto extent = [&](const jpi_kv_cache* c) {
        return (size_t)elem(h) * (size_t)((caches > 1 ? (caches - 1) * c->cache_stride : 0) +
                                          (c->rows > 1 ? (c->rows - 1) * c->row_stride : 0) +
                                          (h->K > 1 ? (h->K - 1) * c->head_stride : 0) +
                                          (layers > 1 ? (layers - 1) * c->layer_stride : 0) + h->D);
    };
    auto overlap = [](const void* a, size_t na, const void* b, size_t nb) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
        return x < y + nb && y < x + na;
    };
    const bool same = src->k == dst->k && src->v == dst->v && src->rows == dst->rows && w == w_out &&
                      (caches == 1 || src->cache_stride == dst->cache_stride) &&
                      (src->rows == 1 || src->row_stride == dst->row_stride) &&
                      (h->K == 1 || src->head_stride == dst->head_stride) &&
                      (layers == 1 || src->layer_stride == dst->layer_stride);
    const size_t ns = extent(src), nd = extent(dst);
    const size_t wn = (size_t)layers * caches * h->K * sizeof(float);
    if (!same && (overlap(src->k, ns, dst->k, nd) || overlap(src->v, ns, dst->v, nd) || overlap(src->k, ns, dst->v, nd) ||
                  overlap(src->v, ns, dst->k, nd) || overlap(w, wn * src->rows, w_out, wn * dst->rows)))
        return fail(JPI_ERR_INVALID_ARG, "dst (with w_out) must be src itself or not overlap it");
    return launch_kv_evict(h, *src, w, length, layers, caches, keep, sink, recent, *dst, w_out, length_out, kept,
                           (cudaStream_t)stream);
}

JPI_API jpi_status jpi_kv_device_status(jpi_kv_handle* h) {
    clear_error();
    JPI_TRY(check_handle(h));
    JPI_CUDA_TRY(cudaDeviceSynchronize());
    int err = 0;
    JPI_CUDA_TRY(cudaMemcpy(&err, h->dev_err, sizeof(int), cudaMemcpyDeviceToHost));
    if (err != DEV_OK) {
        JPI_CUDA_TRY(cudaMemset(h->dev_err, 0, sizeof(int)));
        return fail(JPI_ERR_DEVICE_TIMEOUT, "device-side error code %d (bounded wait gave up)", err);
    }
    return JPI_OK;
}

JPI_API jpi_status jpi_kv_memory_usage(const jpi_kv_handle* h, long long* bytes) {
    clear_error();
    if (!h || !bytes) return fail(JPI_ERR_INVALID_ARG, "NULL argument");
    *bytes = (long long)h->device_bytes;
    return JPI_OK;
}

}  // extern "C"
