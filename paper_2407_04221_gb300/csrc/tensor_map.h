// tensor_map.h -- tensor maps for TMA copies (host).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "autoverse.h"

namespace av {

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder, or NULL where there is none.
inline EncodeTiled map_encoder()
{
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) !=
                cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return (EncodeTiled) nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

// dims, box: innermost first; strides of the outer dims, in elements.  Boxes
// are as wide as the swizzle: 128 bytes, or 64.
inline bool make_map(CUtensorMap *map, int dtype, const void *p, int rank, const int64_t *dims, const int64_t *strides,
                     const int *box, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B)
{
    const int64_t e = dtype == AV_F32 ? 4 : 2;
    cuuint64_t d[5], s[4];
    cuuint32_t b[5], one[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) {
        d[i] = (cuuint64_t)dims[i];
        b[i] = (cuuint32_t)box[i];
        if (i > 0)
            s[i - 1] = (cuuint64_t)(strides[i - 1] * e);
    }
    const CUtensorMapDataType type = dtype == AV_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : dtype == AV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const EncodeTiled encode = map_encoder();
    return encode && encode(map, type, (cuuint32_t)rank, const_cast<void *>(p), d, s, b, one,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace av
