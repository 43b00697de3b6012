// The kernels of jpi_kv_attend: sides with many query rows on tensor-core tiles (kv_attend_t5.cu), the others in
// kv_attend.cu.
#pragma once
#include "kv.h"

namespace jpi {

jpi_status kv_tiles_prepare(jpi_kv_handle* h);
// Key splits (at most `room`) of the sides, prefix and own rows, that take the tiles; 0: not that side.
void kv_tiles_plan(const jpi_kv_handle* h, const KvCall& c, long long room, int splits[2]);
// Parts part0[side] .. + splits[side] - 1 of the call's: `po` [parts][rows][D] and `pml` [rows][parts] (m unscaled, l).
// With `early` it starts while the kernel before it runs, and ends after that.
jpi_status launch_kv_tiles_t5(jpi_kv_handle* h, const KvCall& c, const int splits[2], const int part0[2], float* po, float2* pml,
                              int parts, bool early, cudaStream_t st);

}  // namespace jpi
