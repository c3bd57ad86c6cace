// The gated feed-forward block, shared definitions.  With x [m,k], Wg and Wu [f,k] (rows with strides):
//     G = x Wg^T,  U = x Wu^T,  h = D act(G) U                      (elementwise products)
//     e = D dh,  dU = e act(G),  dG = e U act'(G)
//     dx = dG Wg + dU Wu,  dWg = dG^T x,  dWu = dU^T x
// D is the dropout factor of an element (dropout.cuh).  Nothing of the forward pass but its inputs is kept: the
// backward pass computes G and U again.  dG and dU live in the workspace between the two kernels of the backward
// pass, in the element type: both products take their operands in that type.
#pragma once

#include <cmath>

#include "dropout.cuh"
#include "elements.cuh"
#include "zvc_common.cuh"

namespace cdma {

struct FfnProblem {
    const void *x, *wg, *wu, *dh;
    void *h, *dx, *dwg, *dwu;          // dx, and the pair dwg and dwu, may be null
    uint64_t ld_x, ld_wg, ld_wu, ld_h; // ld_h: of h or of dh
    uint64_t ld_dx, ld_dw;
    uint32_t m, k, f;
    int dtype, activation;
    DropoutSpec drop;
    uint64_t* ws;                      // result words, then what the path needs
    uint64_t result_bytes;
};

constexpr uint64_t kFfnWsHeader = 256;   // bytes in front of the rest of the workspace

// act(g) and its slope.  A ReLU keeps NaNs and lets a gradient through where it kept its input, as the fused ReLU of
// the codec does.  FAST, for results of 2-byte types: the exponential and the quotient by the hardware's
// approximations, a few units of 2^-22 off, where the result is rounded at 2^-9 or 2^-12.
template <bool FAST>
__device__ __forceinline__ float logistic(float g) {
    return FAST ? __fdividef(1.0f, 1.0f + __expf(-g)) : 1.0f / (1.0f + expf(-g));
}
template <int ACT, bool FAST>
__device__ __forceinline__ float activate(float g) {
    if (ACT == CDMA_ACT_RELU) return g > 0.0f || g != g ? g : 0.0f;
    if (ACT == CDMA_ACT_SILU) return g * logistic<FAST>(g);
    return g * normcdff(g);
}
template <int ACT, bool FAST>
__device__ __forceinline__ void activate_slope(float g, float* a, float* slope) {
    if (ACT == CDMA_ACT_RELU) {
        const bool on = g > 0.0f || g != g;
        *a = on ? g : 0.0f;
        *slope = on ? 1.0f : 0.0f;
    } else if (ACT == CDMA_ACT_SILU) {
        const float s = logistic<FAST>(g);
        *a = g * s;
        *slope = s * (1.0f + g * (1.0f - s));
    } else {
        const float cdf = normcdff(g);
        *a = g * cdf;
        *slope = cdf + g * (0.3989422804014327f * (FAST ? __expf(-0.5f * g * g) : expf(-0.5f * g * g)));
    }
}

// Elementwise ends of the two passes; `keep` is the dropout bit of the element.
template <int ACT, bool FAST>
__device__ __forceinline__ float gated_value(float g, float u, bool keep, float scale) {
    return keep ? activate<ACT, FAST>(g) * u * scale : 0.0f;
}
template <int ACT, bool FAST>
__device__ __forceinline__ void gated_gradients(float g, float u, float dh, bool keep, float scale, float* dg, float* du) {
    float a, slope;
    activate_slope<ACT, FAST>(g, &a, &slope);
    const float e = dh * scale;
    *du = keep ? e * a : 0.0f;
    *dg = keep ? e * u * slope : 0.0f;
}

// Forward pass of few rows: of 2-byte elements with strides that TMA takes (gated_ffn_stream.cu) ...
constexpr uint64_t kFewRows = 128;
cudaError_t launch_ffn_stream(const FfnProblem& p, const LaunchCtl& ctl, cudaStream_t stream);
// ... and of 4-byte elements (gated_ffn_rows.cu).
constexpr uint64_t kFewRows4 = 8;
cudaError_t launch_ffn_rows(const FfnProblem& p, const LaunchCtl& ctl, cudaStream_t stream);
// Any number of rows (gated_ffn_mma.cu).
uint64_t ffn_mma_workspace(uint64_t m, uint64_t k, uint64_t f, uint64_t ld_x, uint64_t ld_wg, uint64_t ld_wu, int dtype, bool backward);
cudaError_t launch_ffn_mma(const FfnProblem& p, bool backward, const LaunchCtl& ctl, cudaStream_t stream);

}  // namespace cdma
