// The expert's use of the KV-cache operators: attention of several requests over one stored prefix, the weights its
// keys receive, eviction and extension of the store (jpi_share_prefix and what follows it in include/jpi.h).
#pragma once
#include "kv.h"

namespace jpi {

// What these calls need beside the handle's own buffers, allocated by the first of them.
struct ExpertKv {
    jpi_kv_handle* kv = nullptr;
    int* seen = nullptr;       // [maxB][maxS] suffix keys each suffix token sees
    int* len = nullptr;        // [maxB] prefix lengths
    int* position = nullptr;   // [maxB][maxP] of appended tokens, and the rows they go to
    int* row = nullptr;
    int* kept = nullptr;       // [L][maxB][maxP]
    float* lse = nullptr;      // [maxMt][H]
    // Rotary positions past the expert's table: [maxS][D / 2] (cos, sin) of those that follow the prefix, and the first of them.
    float2* rope = nullptr;
    int* start = nullptr;
};

jpi_status expert_kv_create(jpi_handle* h, ExpertKv* e);
void expert_kv_destroy(ExpertKv* e);
// Fills `seen` and `len` for B requests of C actions, `share` to a prefix.
jpi_status expert_kv_fill(jpi_handle* h, const ExpertKv& e, int B, int C, int share, cudaStream_t st);
// The attention of layer l (o from q and the store); with w, also w [B / share][P] = decay w + weights.
jpi_status expert_kv_attention(jpi_handle* h, const ExpertKv& e, int l, int B, int C, int share, float* w, float decay,
                               cudaStream_t st);
jpi_status expert_kv_evict(jpi_handle* h, const ExpertKv& e, float* w, int keep, int sink, int recent, int* kept, cudaStream_t st);
// Fills `rope` from `start` for the suffix of C actions.
jpi_status expert_kv_rope(jpi_handle* h, const ExpertKv& e, int C, cudaStream_t st);
// `tokens` rows behind the cur_prefix ones of every layer, keys coded for positions from `position` on; `start` follows them.
jpi_status expert_kv_append(jpi_handle* h, const ExpertKv& e, const void* const* k_layers, const void* const* v_layers, int tokens,
                            int position, cudaStream_t st);

}  // namespace jpi
