// Tensor maps of the tensor copies, encoded on the host.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace bigcn {

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder of tensor maps (the library links no driver); nullptr without one.
inline EncodeTiled encoder() {
    static const EncodeTiled fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault,
                                             &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}

// A map of `rows` rows of `width` elements, boxes of box x box_rows; or, with part_bytes, of rows
// of `parts` parts of `width` elements, box_parts of which are in a box.
inline bool encode_map(CUtensorMap *map, CUtensorMapDataType type, const void *base, int64_t width,
                       int64_t rows, int64_t row_bytes, int box, int box_rows, bool swizzle,
                       int64_t parts = 1, int64_t part_bytes = 0, int box_parts = 1) {
    const EncodeTiled fn = encoder();
    if (!fn) return false;
    const cuuint64_t dims[3] = {cuuint64_t(width), cuuint64_t(rows), cuuint64_t(parts)};
    const cuuint64_t strides[2] = {cuuint64_t(row_bytes), cuuint64_t(part_bytes)};
    const cuuint32_t boxes[3] = {cuuint32_t(box), cuuint32_t(box_rows), cuuint32_t(box_parts)};
    const cuuint32_t steps[3] = {1, 1, 1};
    return fn(map, type, part_bytes ? 3 : 2, const_cast<void *>(base), dims, strides, boxes, steps,
              CU_TENSOR_MAP_INTERLEAVE_NONE,
              swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace bigcn
