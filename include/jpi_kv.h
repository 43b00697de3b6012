/*
 * jpi_kv.h — C-ABI of the KV-cache operators: what a program does with a cache of keys and values
 * around the handles of jpi.h and jpi_prefill.h.
 *
 * Paper passages this interface follows:
 *   - App. A ("Model Architecture of pi series Models"): every layer's keys and values are cached
 *     and attended over by queries that come later (the action expert's, over the LLM's cache).
 *   - Sec. 4.3 ("System Design"): intermediate buffers stay on the GPU, and nothing a call does
 *     depends on a host copy: lengths and rows are read from device memory, so that one captured
 *     graph serves a growing cache.
 * The operators themselves (rotary coding of parts and scalings of long contexts, norms of heads, one prefix for
 * many requests, windows, caches in 8 bits, eviction by accumulated attention weight) are no part of the paper.
 *
 *   jpi_kv_append         rotary coding of new queries and keys, keys and values written into the cache
 *   jpi_kv_append_normed  the same after a norm of each head's queries and keys
 *   jpi_kv_attend         attention of a batch over shared prefixes and each request's own rows
 *   jpi_kv_attend_window  attention over the newest rows before each token and a few first ones
 *   jpi_kv_weigh          the attention weight each cached key received, accumulated
 *   jpi_kv_evict          the rows with the most of it kept, in order, the others dropped
 *   jpi_kv8_append        new tokens into a cache held in 8 bits, with a scale for each block of rows and head
 *   jpi_kv8_attend        attention over such a cache, its window included
 *
 * A jpi_kv_handle fixes the attention's geometry, its rotary coding and the maxima of a call, and
 * owns the workspace. Caches belong to the caller: the expert's store (jpi_prefix_kv_ptr), the
 * destinations of jpi_prefill_run, or any buffers of the layout below.
 *
 * Conventions are those of jpi.h: every entry point returns a jpi_status, checks its arguments on
 * the host before anything is enqueued, never aborts, and leaves its message in jpi_last_error().
 * Calls are asynchronous on `stream` and may be captured; a handle is used from one host thread
 * and one stream at a time, and graphs captured from one handle share its workspace, so their
 * replays may not overlap. The calling thread's current device must be the handle's (else
 * JPI_ERR_INVALID_ARG). "Device pointer" means memory of that device.
 * Elements are bf16 in JPI_BF16 mode and fp32 in JPI_FP32 mode ("E" below). Data pointers are
 * 16-byte aligned and strides multiples of 16 bytes.
 */
#ifndef JPI_KV_H
#define JPI_KV_H

#include "jpi.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct jpi_kv_handle jpi_kv_handle;

typedef enum jpi_rope_layout {
    JPI_ROPE_HALF = 0,         /* pair i is elements i and i + dim / 2                            */
    JPI_ROPE_INTERLEAVED = 1   /* pair i is elements 2 i and 2 i + 1                              */
} jpi_rope_layout;

typedef enum jpi_rope_scaling {
    JPI_ROPE_PLAIN = 0,     /* theta_i = base^(-2 i / dim)                                        */
    JPI_ROPE_LINEAR = 1,    /* theta_i / factor                                                   */
    JPI_ROPE_NTK = 2,       /* base * factor^(dim / (dim - 2)) in place of base                   */
    JPI_ROPE_BY_PARTS = 3   /* (1 - g) theta_i / factor + g theta_i, g = clamp((r - low) /        */
                            /* (high - low), 0, 1), r = original theta_i / (2 pi): pairs that     */
                            /* turn less than `low` times over `original` positions are           */
                            /* interpolated, those that turn more than `high` times are not       */
} jpi_rope_scaling;

/* Rotary coding: y1 = m (x1 cos a - x2 sin a), y2 = m (x2 cos a + x1 sin a), a = position theta_i,
 * for pair i of the first `dim` elements of a head; the others pass through. */
typedef struct jpi_kv_rope {
    int dim;          /* even, 2 .. head_dim                                                      */
    int layout;       /* jpi_rope_layout                                                          */
    int scaling;      /* jpi_rope_scaling                                                         */
    int original;     /* context length of JPI_ROPE_BY_PARTS, >= 1                                */
    float base;       /* >= 1                                                                     */
    float factor;     /* >= 1 (JPI_ROPE_NTK: dim >= 4)                                            */
    float low, high;  /* JPI_ROPE_BY_PARTS: low < high                                            */
    float mscale;     /* m above, > 0 (1: a rotation)                                             */
} jpi_kv_rope;

typedef struct jpi_kv_config {
    int n_heads;      /* H query heads, a multiple of n_kv_heads                                  */
    int n_kv_heads;   /* Hk; query head h reads KV head h / (H / Hk)                              */
    int head_dim;     /* D, at most 256; a multiple of 8 (JPI_BF16) or 4 (JPI_FP32)               */
    int max_batch;    /* most requests per call                                                   */
    int max_tokens;   /* most new tokens of one request per call                                  */
    float scale;      /* of the attention scores, 2^-32 .. 2^32; 0: 1 / sqrt(D)                   */
    jpi_precision precision;
} jpi_kv_config;

/* `n` caches of `rows` rows: element d of KV head h in row r of cache c is at
 * base + c cache_stride + r row_stride + h head_stride + d (elements), for k and v alike.
 * [c][rows][Hk][D] and [c][Hk][rows][D] are both such caches. A stride of a dimension of size 1 is
 * not used; the others are positive. */
typedef struct jpi_kv_cache {
    void *k, *v;
    long long cache_stride, row_stride, head_stride;
    long long layer_stride;   /* jpi_kv_evict: layer l is l layer_stride elements further on        */
    int rows;                 /* rows of each cache that a call may touch                           */
} jpi_kv_cache;

/* Checks the shapes, allocates the workspace for the maxima and tabulates the rotary coding (NULL:
 * none; append then copies). Synchronous; the only call that allocates. On failure *out is NULL. */
JPI_API jpi_status jpi_kv_create(const jpi_kv_config* cfg, const jpi_kv_rope* rope, jpi_kv_handle** out);
/* The environment read here: JPI_KV_TILES=0 / 1 keeps jpi_kv_attend and jpi_kv_weigh on the kernels for few query rows,
 * or on the tensor-core tiles wherever those fit, for the handle's lifetime (results agree to rounding: see
 * jpi_kv_attend for that of the probabilities). The workspace is attention's and has the same size whichever calls are made:
 * (2 max_batch max_tokens H + 512 SMs) rows of head_dim + 2 fp32 numbers, 80 MB at least for heads of 256 on 152 SMs. */
JPI_API jpi_status jpi_kv_destroy(jpi_kv_handle* h);   /* NULL is a no-op */

/*
 * Rotary coding and cache write of batch x tokens new tokens.
 *   q, k, v:   device E; token (b, t)'s head h at base + (b tokens + t) stride + h D, H heads of q and
 *              Hk of k and v. v may be NULL (keys only: keys of a cache coded in place or moved).
 *              q may be NULL (with q_out NULL: no queries); k NULL: queries only.
 *   position:  device int [batch][tokens], any value (negative: the rotation backwards).
 *   row:       device int [batch][tokens], the row of cache b that takes the token. A row outside
 *              0 .. cache->rows - 1 marks padding: nothing is written for that token, its q_out
 *              included. A row that several tokens of one request name is left with elements of any of
 *              them, mixed and not the same from call to call; no other row is touched by them.
 *   q_out:     device E [batch][tokens][H][D], the coded queries (may alias q where q is contiguous).
 *   cache:     `batch` caches; its k (and v) may be where k (and v) point to, the same rows at the
 *              same addresses.
 * Angles are within 2^-26 + |position| 2^-53 turns (2^-26: the phase as an fp32 number; 2^-53: the table, whose
 * entries are computed in 64-bit floating point). Sums in fp32, one rounding to E.
 */
JPI_API jpi_status jpi_kv_append(jpi_kv_handle* h, const void* q, long long q_stride, const void* k,
                                 long long k_stride, const void* v, long long v_stride, const int* position,
                                 const int* row, int batch, int tokens, void* q_out, const jpi_kv_cache* cache,
                                 void* stream);

/*
 * Attention of batch x tokens query tokens. The requests come in `groups` runs of batch / groups
 * (groups divides batch); request b's keys are the first prefix_len[g] rows of prefix g of its run,
 * shared by the whole run and read once for it, and then rows of its own cache: query token (b, t)
 * sees rows 0 .. seen[b][t] - 1 of it (causal order, a state token that sees itself only, padding
 * that sees nothing: whatever the counts say).
 *   q:           device E, as in jpi_kv_append
 *   prefix:      `groups` caches, or NULL (prefix_len is then NULL too, groups 1)
 *   prefix_len:  device int [groups]; taken as 0 .. prefix->rows
 *   own:         `batch` caches, or NULL (seen is then NULL too)
 *   seen:        device int [batch][tokens]; taken as 0 .. own->rows
 *   out:         device E [batch][tokens][H][D]
 *   lse:         device fp32 [batch][tokens][H], log of the sum of exp(score), or NULL
 * A query that sees no key gets zeros and -infinity (as one all of whose scores are -infinity). A NaN score,
 * of a NaN in the query or in a key that it sees, makes out and lse NaN, and so the weights that jpi_kv_weigh
 * forms with them. An infinite value that a query sees makes the element infinite, NaN where both signs meet or where
 * its weight is below the least that fp32 holds. Nothing in rows that a query does not see reaches it, infinities and
 * NaN included. Scores, softmax and sums in fp32; results do not depend on the run. In JPI_BF16 mode the
 * probabilities enter the second product as bf16: calls of many query rows on the same keys, which take the 128-row
 * tensor-core tiles, round each once (off by at most 2^-8 of itself, so an element by at most 2^-8 of the sum of
 * p |v|); the others carry what the rounding left as a second term (2^-16). A handle made with JPI_KV_TILES=0 always has both
 * terms, at the row kernels' speed.
 */
JPI_API jpi_status jpi_kv_attend(jpi_kv_handle* h, const void* q, long long q_stride, int batch, int tokens,
                                 const jpi_kv_cache* prefix, int groups, const int* prefix_len,
                                 const jpi_kv_cache* own, const int* seen, void* out, float* lse, void* stream);

/*
 * Accumulated attention weight: out[key] = decay * in[key] + sum of exp(score - lse) over the
 * query tokens and heads that see the key (of the KV head's own H / Hk query heads). Arguments as in
 * jpi_kv_attend, with lse its result; only the caches' keys are read.
 *   prefix_in, prefix_out:  device fp32 [groups][Hk][prefix->rows]; in may be NULL (taken as zeros, as
 *              decay 0 takes it) or the same buffer as out.
 *   own_in, own_out:        device fp32 [batch][Hk][own->rows], likewise.
 * Entries of rows that hold no key (from prefix_len, or the largest seen count of the request,
 * on) are left as they are.
 */
JPI_API jpi_status jpi_kv_weigh(jpi_kv_handle* h, const void* q, long long q_stride, const float* lse, int batch,
                                int tokens, const jpi_kv_cache* prefix, int groups, const int* prefix_len,
                                const jpi_kv_cache* own, const int* seen, float decay, const float* prefix_in,
                                float* prefix_out, const float* own_in, float* own_out, void* stream);

/*
 * Eviction: of the first length[c] rows (taken as 0 .. src->rows) of each cache c, `keep` stay
 * (all, where there are no more): the first `sink`, the last `recent`, and of the others those with
 * the largest weight, ties to the lowest row, NaN below everything else. Every layer, cache and KV
 * head chooses by its own weights. The kept rows move to the front in their order, keys, values and
 * weights alike.
 *   src:      `layers` x `caches` caches (layer_stride apart)
 *   w:        device fp32 [layers][caches][Hk][src->rows]
 *   length:   device int [caches]
 *   dst:      where the kept rows go: src itself (in place: the same pointers, strides and rows) or
 *             caches of at least `keep` rows that do not overlap it
 *   w_out:    device fp32 [layers][caches][Hk][dst->rows]; w itself where dst is src
 *   length_out: device int [caches], min(length, keep); may be `length`
 *   kept:     device int [layers][caches][Hk][keep], the rows of src that stay, ascending; -1 behind them
 * sink + recent <= keep <= src->rows. Rows and weights of dst behind the kept ones are left as they
 * are. Keys stay coded for the positions they had.
 */
JPI_API jpi_status jpi_kv_evict(jpi_kv_handle* h, const jpi_kv_cache* src, const float* w, const int* length,
                                int layers, int caches, int keep, int sink, int recent, const jpi_kv_cache* dst,
                                float* w_out, int* length_out, int* kept, void* stream);

/* Norms of a head's queries and keys before their rotary coding: x / sqrt(mean(x^2) + eps) * weight, over the D
 * elements of each head. */
typedef struct jpi_kv_norm {
    const float *q_weight, *k_weight;   /* device fp32 [D], 4-byte aligned; NULL: ones                */
    float eps;                          /* 2^-126 or more, finite                                    */
} jpi_kv_norm;

/*
 * jpi_kv_append after a norm of each head of q and k, in one pass; v is copied. Arguments and what is written as there.
 * Squares are summed in fp32 (where the mean of a head's squares with eps passes 1e38 they are summed again at 2^-70 of its values,
 * and eps is taken at 2^-140, so that finite values give finite norms); everything up to the one rounding to E is fp32.
 */
JPI_API jpi_status jpi_kv_append_normed(jpi_kv_handle* h, const void* q, long long q_stride, const void* k,
                                        long long k_stride, const void* v, long long v_stride, const jpi_kv_norm* norm,
                                        const int* position, const int* row, int batch, int tokens, void* q_out,
                                        const jpi_kv_cache* cache, void* stream);

/*
 * Attention over a window: query token (b, t) sees of cache b's rows before seen[b][t] the first `sink` ones and the
 * last `window` ones, rows r < seen with r < sink or r >= seen - window.
 *   cache:   `batch` caches
 *   seen:    device int [batch][tokens]; taken as 0 .. cache->rows (0: padding, which sees nothing)
 *   window:  >= 1;  sink: >= 0
 * q, out, lse, empty rows, NaN and infinities as in jpi_kv_attend; rows outside a token's window are rows that it does not
 * see. The tokens of a request whose rows run together (8 rows, tokens x heads of a KV head, or 128 on the tiles) read the first
 * `sink` rows and all from the lowest row of their windows to their largest count, the tiles in whole blocks of 64: for tokens that
 * follow one another the work goes by the windows, not by the cache's length, but tokens of one call with counts far apart also
 * cost what lies between their windows. In JPI_BF16 mode the probabilities enter the second product as there: calls of many query rows on
 * the 128-row tiles round each to bf16 once, the others carry what the rounding left. JPI_KV_TILES holds here too. Sums of p v are formed at up to
 * 2^24 times their size (2^8 outside the tiles): finite values of 2^100 and more may come out infinite. A handle's first call here or of
 * jpi_kv8_attend looks up what the device holds of their kernels (2 ms in a process, 0.4 ms for a further head width); it may be captured.
 */
JPI_API jpi_status jpi_kv_attend_window(jpi_kv_handle* h, const void* q, long long q_stride, int batch, int tokens,
                                        const jpi_kv_cache* cache, const int* seen, int window, int sink, void* out,
                                        float* lse, void* stream);

/*
 * `n` caches of `rows` rows in 8 bits: element d of KV head h in row r of cache c is an e4m3 number at
 * base + c cache_stride + r row_stride + h head_stride + d (bytes; strides multiples of 16 as the base is), times
 * 2^(s - 127) with s the byte (e8m0) of its block of `block` rows and head, scale[c][h][r / block], contiguous
 * [n][Hk][ceil(rows / block)]. A scale of 255 is NaN and makes the block's elements NaN. head_dim is a multiple of 16
 * (else JPI_ERR_UNSUPPORTED).
 */
typedef struct jpi_kv8_cache {
    void *k, *v;
    unsigned char *k_scale, *v_scale;
    long long cache_stride, row_stride, head_stride;
    int rows;
    int block;        /* 16, 32 or 64 rows                                                           */
} jpi_kv8_cache;

/*
 * Rotary coding, with `norm` (may be NULL: none) after norms as in jpi_kv_append_normed, and the write into 8-bit caches:
 * token t < count[b] of request b goes to row start[b] + t of cache b.
 *   start:  device int [batch], the rows that cache b holds before the call; what later rows hold is taken as nothing. A
 *           start outside 0 .. cache->rows - 1 marks a request of padding only.
 *   count:  device int [batch], taken as 0 .. tokens; NULL: tokens. Later tokens, and those that would pass the last row, are
 *           padding: nothing is written for them, their q_out included.
 * A block that holds no row before `start` gets the least scale 2^k, -126 <= k, at which its new elements' magnitudes are at
 * most 448 (in the block, of one head; keys and values by themselves). One that does keeps its scale or has it raised to
 * that, and its rows before `start` are rounded again to the new scale: a step of a power of two, exact but for
 * elements below 2^-6 of the new scale, which move by at most 2^-10 of it. Each new element is rounded once, from fp32 to the nearest code
 * (off by at most 2^-4 of itself, or 2^-10 of the scale). Infinities and NaN do not count for the scale and are held
 * as NaN. Rows of a block behind the new ones are left as they are; a scale of 255 under rows before `start` stays.
 * k and v go together. Everything else as in jpi_kv_append.
 */
JPI_API jpi_status jpi_kv8_append(jpi_kv_handle* h, const void* q, long long q_stride, const void* k, long long k_stride,
                                  const void* v, long long v_stride, const jpi_kv_norm* norm, const int* position,
                                  const int* start, const int* count, int batch, int tokens, void* q_out,
                                  const jpi_kv8_cache* cache, void* stream);

/*
 * Attention over 8-bit caches: query token (b, t) sees rows 0 .. seen[b][t] - 1 of cache b, with window >= 1 as in
 * jpi_kv_attend_window (0: all of them, and `sink` is not used). q, out and lse are as in jpi_kv_attend, of the handle's type; so
 * are empty rows, and NaN in what a query sees.
 * Scores, softmax and sums in fp32, codes and scales taken as they are. JPI_BF16 mode: queries enter the first product as fp16,
 * scaled by a power of two (bf16's eight bits whole; an element below 2^-14 of its head's largest is off by at most 2^-25 of
 * that), the probabilities the second as fp16 (each off by at most 2^-11 of itself, or 2^-28 of what the largest value of the
 * blocks seen would weigh). JPI_KV_TILES holds here too, and what jpi_kv_attend_window says of the rows that are read. Sums of p v are formed at
 * up to 2^11 times their size (2^8 outside the tiles): finite values of 2^100 and more may come out infinite.
 */
JPI_API jpi_status jpi_kv8_attend(jpi_kv_handle* h, const void* q, long long q_stride, int batch, int tokens,
                                  const jpi_kv8_cache* cache, const int* seen, int window, int sink, void* out,
                                  float* lse, void* stream);

/* Synchronises the device and reports device-side errors of earlier calls, as jpi_device_status. */
JPI_API jpi_status jpi_kv_device_status(jpi_kv_handle* h);

/* Bytes of device memory the handle holds. */
JPI_API jpi_status jpi_kv_memory_usage(const jpi_kv_handle* h, long long* bytes);

#ifdef __cplusplus
}
#endif

#endif /* JPI_KV_H */
