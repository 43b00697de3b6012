// Bulk tensor maps of a cache's keys or values (kv_maps.cu): four dimensions, the elements of a head and then heads,
// rows and caches by ascending stride, those of size 1 last.
#pragma once
#include "kv.h"
#include "../ptx.h"

namespace jpi {

struct KvMapDims {
    uint64_t size[3], stride[3];              // stride in bytes
    int at_head = 0, at_row = 0, at_cache = 0;   // which outer dimension is which
};

// The dimensions of `n` caches of this side, K heads of D bf16 elements. False where the strides are not those that
// maps are documented for (each a multiple of the one before, below 2^40 bytes).
bool kv_map_dims(const KvSide& s, int K, int D, int n, KvMapDims* m);
// Map with boxes of 64 elements x `rows` rows, 128-byte swizzle, zeros past the ends.
bool kv_make_map(const KvMapDims& m, const void* base, int D, int rows, CUtensorMap* map);

#ifdef __CUDACC__
// Box at element x, head, row and cache; m's positions in `at` = (head, row, cache).
__device__ __forceinline__ void kv_load_box(void* dst, const void* tmap, uint64_t* bar, int x, int3 at, int head, int row,
                                            int cache) {
    auto coord = [&](int dim) { return dim == at.y ? row : dim == at.x ? head : cache; };
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(ptx::smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(coord(0)), "r"(coord(1)), "r"(coord(2)), "r"(ptx::smem_u32(bar))
        : "memory");
}
#endif

}  // namespace jpi
