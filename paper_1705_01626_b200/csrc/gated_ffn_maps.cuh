// Operands of the matrix units as TMA sees them.
#pragma once

#include "gated_ffn.cuh"
#include "tensor_map.h"

namespace cdma {

inline uint64_t pitch_of(uint64_t cols) { return (cols + 63) & ~63ull; }
inline uint32_t tiles_of(uint64_t n, uint32_t t) { return static_cast<uint32_t>((n + t - 1) / t); }

struct Matrix {
    const void* p;
    uint64_t rows, cols, ld;
    uint32_t planes;
};

// Boxes of 64 columns (128 bytes, swizzled) and `lines` rows.  The stride of a single row is free.
inline bool make_operand_map(CUtensorMap* map, const Matrix& m, int dtype, uint32_t lines) {
    const uint64_t ld = m.rows > 1 ? m.ld : pitch_of(m.cols);
    return encode_matrix_map(map, dtype == CDMA_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p,
                             m.rows, m.cols, ld, m.planes, m.rows * ld, 64, lines, CU_TENSOR_MAP_SWIZZLE_128B);
}

}  // namespace cdma
