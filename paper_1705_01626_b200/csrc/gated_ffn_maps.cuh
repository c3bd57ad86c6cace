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

// 4-byte elements go to the matrix units as three bf16 planes, x = high + middle + low, 8 bits each.  The six products of
// planes that reach 2^-24 of the whole are taken, the small ones first.
template <typename T> struct Planes { static constexpr uint32_t count = 1, products = 1; };
template <> struct Planes<float> { static constexpr uint32_t count = 3, products = 6; };
// Planes of A and of B in the parts of the reduction (4 bits each, the first part lowest).
constexpr uint32_t kPlaneOfA = 0x010120u, kPlaneOfB = 0x001102u;

// The three bf16 planes of a float, cut off so that the two upper ones never round up to infinity.  What is not
// finite goes into the first plane alone.
__device__ __forceinline__ void split3(float v, uint32_t (&planes)[3]) {
    const uint32_t bits = __float_as_uint(v);
    const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
    const uint32_t high = finite || (bits & 0x007fffffu) == 0 ? bits & 0xffff0000u : 0x7fc00000u;
    const float rest = finite ? v - __uint_as_float(high) : 0.0f;
    const uint32_t middle = __float_as_uint(rest) & 0xffff0000u;
    planes[0] = high >> 16;
    planes[1] = middle >> 16;
    planes[2] = pack2<__nv_bfloat16>(rest - __uint_as_float(middle), 0.0f) & 0xffffu;
}

// Boxes of 64 columns (128 bytes, swizzled) and `lines` rows.  The stride of a single row is free.
inline bool make_operand_map(CUtensorMap* map, const Matrix& m, int dtype, uint32_t lines) {
    const uint64_t ld = m.rows > 1 ? m.ld : pitch_of(m.cols);
    return encode_matrix_map(map, dtype == CDMA_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p,
                             m.rows, m.cols, ld, m.planes, m.rows * ld, 64, lines, CU_TENSOR_MAP_SWIZZLE_128B);
}

// G and U of few rows (gated_ffn_stream.cu) and from them h or, with `grads`, dG and dU there.
cudaError_t launch_ffn_stream(const FfnProblem& p, const Matrix& x, const Matrix& wg, const Matrix& wu, void* grads, uint64_t ld_grad,
                              const LaunchCtl& ctl, cudaStream_t stream);

}  // namespace cdma
