// Tensor maps over a pool's pages.
#pragma once
#include <cuda.h>

#include "plc_pages.cuh"

namespace plc {
namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() {
    static const EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess
                   ? reinterpret_cast<EncodeTiledFn>(f) : nullptr;
    }();
    return fn;
}

// A layer's keys and values in boxes of 64 components by `box` positions of one page (a divisor of its size, a multiple of eight).  box_dim: what dimensions 1 .. 4 of
// the map are (0 slot, 1 head, 2 page, 3 key or value).  False where the pool has no such boxes: vectors of 32 components (a box row would be half a shared
// memory row), strides that are not positive or not multiples of each other.
bool page_boxes(const PoolDev& p, int layer, bool bf16, int box, CUtensorMap* map, int* box_dim) {
    if (p.d < 64) return false;
    const int64_t stride[4] = {p.sp, p.sh, p.spage, p.skv};
    const cuuint64_t extent[4] = {(cuuint64_t)p.page_pos, (cuuint64_t)p.H, (cuuint64_t)p.n_pages, 2};
    int order[4] = {0, 1, 2, 3};
    for (int i = 0; i < 4; ++i) {
        if (stride[i] <= 0 || stride[i] >= (1ll << 40)) return false;
        for (int j = i; j > 0 && stride[order[j]] < stride[order[j - 1]]; --j) { const int t = order[j]; order[j] = order[j - 1]; order[j - 1] = t; }
    }
    cuuint64_t dims[5] = {(cuuint64_t)p.d}, strides[4];
    cuuint32_t boxes[5] = {64}, ones[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < 4; ++i) {
        dims[i + 1] = extent[order[i]];
        strides[i] = (cuuint64_t)stride[order[i]];
        boxes[i + 1] = order[i] == 0 ? (cuuint32_t)box : 1;
        if (i > 0 && strides[i] % strides[i - 1]) return false;
        box_dim[i] = order[i];
    }
    const EncodeTiledFn fn = encode_tiled_fn();
    return fn && fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5, p.base + (int64_t)layer * p.sl, dims, strides, boxes, ones,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace plc
