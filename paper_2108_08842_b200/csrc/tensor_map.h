// Tensor maps of the products' operands.
#pragma once

#include <cuda.h>

#include "train_host.h"

namespace eden {
namespace {

using EncodeMap = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeMap encode_map()
{
    static const EncodeMap fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) == cudaSuccess &&
                        found == cudaDriverEntryPointSuccess;
        return ok ? (EncodeMap)p : nullptr;
    }();
    return fn;
}

// boxes of a matrix, zeros outside
int encode_tiles(CUtensorMap* map, CUtensorMapDataType type, const void* data, const cuuint64_t (&dims)[2], const cuuint64_t (&strides)[1],
                 const cuuint32_t (&box)[2], CUtensorMapSwizzle swizzle)
{
    const EncodeMap fn = encode_map();
    if (!fn) return EDEN_ERR_CUDA;
    const cuuint32_t unit[2] = {1, 1};
    const CUresult rc = fn(map, type, 2, const_cast<void*>(data), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? EDEN_OK : EDEN_ERR_CUDA;
}

// the largest power of two, up to 32, of which every row's address is a multiple
int row_grain(const void* p, uint64_t stride, size_t size)
{
    const uint64_t bits = (uint64_t)(uintptr_t)p | stride * size | 32;
    return (int)(bits & (0 - bits));
}

}  // namespace
}  // namespace eden
