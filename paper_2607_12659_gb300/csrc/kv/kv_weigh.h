// The prefix side of jpi_kv_weigh on tensor-core tiles of 128 keys x 128 query rows (kv_weigh_t5.cu).
#pragma once
#include "kv.h"

namespace jpi {

jpi_status kv_weigh_prepare(jpi_kv_handle* h);
// Whether the call's prefix side takes that kernel.
bool kv_weigh_tiles(const jpi_kv_handle* h, const KvCall& c);
// With `early` it starts while the kernel before it runs, and ends after that.
jpi_status launch_kv_weigh_t5(jpi_kv_handle* h, const KvCall& c, const float* lse, float decay, const float* in, float* out,
                              bool early, cudaStream_t st);

}  // namespace jpi
