// Bulk tensor maps of a cache (kv_maps.h).

#include "kv_maps.h"

#include <cudaTypedefs.h>

#include <algorithm>

namespace jpi {
namespace {

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        cudaDriverEntryPointQueryResult q;
        void* p = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return (PFN_cuTensorMapEncodeTiled_v12000)p;
    }();
    return fn;
}

}  // namespace

bool kv_map_dims(const KvSide& s, int K, int D, int n, KvMapDims* m) {
    struct Dim {
        long long stride;
        int size, id;
    } d[3] = {{s.hs, K, 0}, {s.rs, s.rows, 1}, {s.cs, n, 2}};
    std::stable_sort(d, d + 3, [](const Dim& x, const Dim& y) {
        if ((x.size > 1) != (y.size > 1)) return x.size > 1;
        return x.size > 1 && x.stride < y.stride;
    });
    long long last = D;   // a multiple of 16 bytes
    for (int i = 0; i < 3; ++i) {
        const long long st = d[i].size > 1 ? d[i].stride : last;
        if ((i > 0 && st % last) || st >= (1ll << 39)) return false;
        last = st;
        m->size[i] = (uint64_t)d[i].size;
        m->stride[i] = (uint64_t)st * 2;
        (d[i].id == 0 ? m->at_head : d[i].id == 1 ? m->at_row : m->at_cache) = i;
    }
    return true;
}

bool kv_make_map(const KvMapDims& m, const void* base, int D, int rows, CUtensorMap* map) {
    auto enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)D, m.size[0], m.size[1], m.size[2]};
    const cuuint64_t strides[3] = {m.stride[0], m.stride[1], m.stride[2]};
    cuuint32_t box[4] = {64, 1, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    box[1 + m.at_row] = (cuuint32_t)rows;
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace jpi
