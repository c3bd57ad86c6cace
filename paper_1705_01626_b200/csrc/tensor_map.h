// TMA descriptors of row-major matrices.
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

namespace cdma {

// The driver's tensor-map encoder, looked up once (no link-time dependency on the driver library).
inline PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    }();
    return fn;
}

// Map of `planes` matrices of rows x cols elements of `size` bytes, `ld` elements from row to row and `plane` from matrix
// to matrix, in boxes of box_cols x box_rows of one plane.  The start and the strides must be multiples of 16 bytes.
// Places outside a matrix read as zero.
inline bool encode_matrix_map(CUtensorMap* map, CUtensorMapDataType type, uint32_t size, const void* p, uint64_t rows, uint64_t cols,
                              uint64_t ld, uint32_t planes, uint64_t plane, uint32_t box_cols, uint32_t box_rows,
                              CUtensorMapSwizzle swizzle) {
    const auto encode = tensor_map_encoder();
    if (encode == nullptr) return false;
    const cuuint64_t dims[3] = {cols, rows, planes}, strides[2] = {ld * size, (planes > 1 ? plane : ld) * size};
    const cuuint32_t box[3] = {box_cols, box_rows, 1}, steps[3] = {1, 1, 1};
    return encode(map, type, 3, const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace cdma
