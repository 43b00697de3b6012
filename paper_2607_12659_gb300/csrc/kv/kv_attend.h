// The kernels of jpi_kv_attend: sides with many query rows on tensor-core tiles (kv_attend_t5.cu), the others in
// kv_attend.cu.
#pragma once
#include "kv.h"

namespace jpi {

// Key splits of the sides, prefix and own rows, that take the tiles (0: not that side), or with `both` of the tiles of
// the requests' rows that take the prefix's keys and the own ones (splits[1]).
struct KvTilesPlan {
    int splits[2] = {0, 0};
    bool both = false;
    bool takes(bool own) const { return splits[own] > 0 || both; }
};

jpi_status kv_tiles_prepare(jpi_kv_handle* h);
// The plan of a call whose parts may be `room` a side.
void kv_tiles_plan(const jpi_kv_handle* h, const KvCall& c, long long room, KvTilesPlan* plan);
// Parts part0[side] .. + splits[side] - 1 of the call's: `po` [parts][rows][D] and `pml` [rows][parts] (m unscaled, l); with
// one part in all the result itself. With `early` it starts while the kernel before it runs, and ends after that.
jpi_status launch_kv_tiles_t5(jpi_kv_handle* h, const KvCall& c, const KvTilesPlan& plan, const int part0[2], float* po,
                              float2* pml, int parts, void* out, float* lse, bool early, cudaStream_t st);

// Joins the parts 0 .. parts - 1 that a call's kernels left in the handle's workspace.
jpi_status launch_kv_combine(const jpi_kv_handle* h, const KvCall& c, int parts, void* out, float* lse, cudaStream_t st);

}  // namespace jpi
