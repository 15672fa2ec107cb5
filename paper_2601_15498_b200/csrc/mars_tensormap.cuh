// Host: tensor maps for tiled TMA loads.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <mutex>

namespace mars {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled()
{
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *sym = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = (EncodeTiledFn)sym;
    });
    return fn;
}

// [rows, columns] row-major with `stride` bytes a row -> boxes of [box_rows x box_columns] elements, 128-byte
// swizzle, zeros outside.  Base and stride are multiples of 16 bytes.
inline bool tensor_map_2d(CUtensorMap *map, CUtensorMapDataType type, const void *ptr, uint64_t rows, uint64_t columns,
                          uint64_t stride, uint32_t box_rows, uint32_t box_columns)
{
    EncodeTiledFn enc = encode_tiled();
    if (!enc) return false;
    cuuint64_t dims[2] = {columns, rows};
    cuuint64_t strides[1] = {stride};
    cuuint32_t box[2] = {box_columns, box_rows};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, type, 2, const_cast<void *>(ptr), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace mars
