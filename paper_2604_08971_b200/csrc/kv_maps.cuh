// Tensor maps of keys and values for the TMA copies of serving attention.
#pragma once
#include <cuda.h>

#include "serving.cuh"
#include "tc_common.cuh"

namespace {

CUtensorMapSwizzle kv_swizzle(int row_bytes) {
    return row_bytes >= 128 ? CU_TENSOR_MAP_SWIZZLE_128B : row_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : row_bytes == 32 ? CU_TENSOR_MAP_SWIZZLE_32B
                                                                                                                        : CU_TENSOR_MAP_SWIZZLE_NONE;
}
// K or V, dense and 16-bit, as boxes of (64 columns at most, box_rows tokens) of (d, token, head, batch); a dimension of stride 0 is one that
// every index shares.
bool make_map_dense(CUtensorMap* tm, const void* ptr, const KvAttendArgs& a, const long long st[3], int box_rows) {
    EncodeTiledFn fn = get_encode_fn();
    if (fn == nullptr) return false;
    const int rb = a.d >= 64 ? 128 : a.d * 2;
    cuuint64_t dims[4] = {(cuuint64_t)a.d, (cuuint64_t)a.Tk, st[1] ? (cuuint64_t)a.Hk : 1, st[0] ? (cuuint64_t)a.B : 1};
    cuuint64_t strides[3] = {(cuuint64_t)(st[2] ? st[2] : 8) * 2, (cuuint64_t)(st[1] ? st[1] : 8) * 2, (cuuint64_t)(st[0] ? st[0] : 8) * 2};
    cuuint32_t box[4] = {(cuuint32_t)rb / 2, (cuuint32_t)box_rows, 1, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(tm, a.dtype == SENTRY_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, kv_swizzle(rb), CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The codes of a cache as boxes of box_rows tokens of (d, all tokens of all heads of all pages).
bool make_map_codes(CUtensorMap* tm, const void* ptr, const KvAttendArgs& a, int box_rows) {
    EncodeTiledFn fn = get_encode_fn();
    if (fn == nullptr) return false;
    cuuint64_t dims[2] = {(cuuint64_t)a.d, (cuuint64_t)a.n_pages * a.Hk * a.page};
    cuuint64_t strides[1] = {(cuuint64_t)a.d};
    cuuint32_t box[2] = {(cuuint32_t)a.d, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, kv_swizzle(a.d),
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
struct KvMaps { CUtensorMap k, v; };

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* tmap, int x, int y, int z, int w, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
                 : "memory");
}

}  // namespace
