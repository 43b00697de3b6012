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

// An ordinary launch, or with `early` one that starts while the kernel before it runs.
template <typename... Params, typename... Args>
jpi_status kv_start(void (*kernel)(Params...), long long grid, int threads, size_t smem, bool early, cudaStream_t st,
                    const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = early ? 1 : 0;
    JPI_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    return JPI_OK;
}

}  // namespace jpi
