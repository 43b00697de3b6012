// The kernels of jpi_kv_attend: the prefix side on tensor-core tiles of 128 query rows (kv_attend_t5.cu), the others
// in kv_attend.cu.
#pragma once
#include "kv.h"

namespace jpi {

jpi_status kv_prefix_prepare(jpi_kv_handle* h);
// Whether the call's prefix side takes that kernel, and then its key splits (at most `room`).
bool kv_prefix_splits(const jpi_kv_handle* h, const KvCall& c, long long room, int* splits);
// Parts 0 .. splits - 1 of the call's: `po` [parts][rows][D] and `pml` [rows][parts] (m unscaled, l). With `early` it starts while
// the kernel before it runs, and ends after that.
jpi_status launch_kv_prefix_t5(jpi_kv_handle* h, const KvCall& c, int splits, float* po, float2* pml, int parts,
                               bool early, cudaStream_t st);

}  // namespace jpi
