// The gated feed-forward block for 4-byte elements, on the ordinary arithmetic units (the matrix units would round the
// operands to 10 or fewer bits), for any stride and size: tiled products with 128 x 128 outputs per block, 8 x 8 per thread, a reduction step of 16 staged through shared memory while the
// next one is on its way into registers.
#include "gated_ffn.cuh"

namespace cdma {
namespace {

constexpr uint32_t kTile = 128, kStep = 16, kThreads = 256, kPitch = kTile + 4;

// A reduction step of an operand, 16 x 128, is 512 groups of four elements that are neighbours in memory: two for
// each thread.  ALONG: neighbours follow each other in the reduction (else across the tile).
template <bool ALONG>
__device__ __forceinline__ void group_of(uint32_t g, uint32_t* line, uint32_t* red) {
    if (ALONG) { *line = g >> 2; *red = (g & 3) * 4; }
    else       { *line = (g & 31) * 4; *red = g >> 5; }
}

// Four neighbours from p on, of which `there` exist.
__device__ __forceinline__ void load4(const float* p, int64_t there, bool vectors, float v[4]) {
    if (vectors && there >= 4) {
        const float4 q = *reinterpret_cast<const float4*>(p);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < there ? p[i] : 0.0f;
}

template <bool ALONG>
__device__ __forceinline__ void store4(float (*s)[kPitch], uint32_t line, uint32_t red, const float v[4]) {
    if (ALONG) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[red + i][line] = v[i];
    } else {
        *reinterpret_cast<float4*>(&s[red][line]) = make_float4(v[0], v[1], v[2], v[3]);
    }
}

struct Shared {
    float a[2][kStep][kPitch], b[2][kStep][kPitch];
};

// acc = A B over `steps` reduction steps; fetch_a / fetch_b(step, group, values) bring one group into registers.
template <bool A_ALONG, bool B_ALONG, typename FA, typename FB>
__device__ __forceinline__ void product(Shared& sh, float (&acc)[8][8], uint32_t steps, FA fetch_a, FB fetch_b) {
    const uint32_t tx = threadIdx.x & 15u, ty = threadIdx.x >> 4;
    float va[2][4], vb[2][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.0f;
    for (uint32_t step = 0; step <= steps; ++step) {
        if (step < steps) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fetch_a(step, threadIdx.x + i * kThreads, va[i]);
                fetch_b(step, threadIdx.x + i * kThreads, vb[i]);
            }
        }
        if (step != 0) {
            float (*a)[kPitch] = sh.a[(step - 1) & 1], (*b)[kPitch] = sh.b[(step - 1) & 1];
#pragma unroll
            for (uint32_t r = 0; r < kStep; ++r) {
                float x[8], y[8];
                *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(&a[r][ty * 4]);
                *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(&a[r][64 + ty * 4]);
                *reinterpret_cast<float4*>(y) = *reinterpret_cast<const float4*>(&b[r][tx * 4]);
                *reinterpret_cast<float4*>(y + 4) = *reinterpret_cast<const float4*>(&b[r][64 + tx * 4]);
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
            }
        }
        if (step < steps) {
            // the buffer written here was last read two steps ago, in front of the previous barrier
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t line, red;
                group_of<A_ALONG>(threadIdx.x + i * kThreads, &line, &red);
                store4<A_ALONG>(sh.a[step & 1], line, red, va[i]);
                group_of<B_ALONG>(threadIdx.x + i * kThreads, &line, &red);
                store4<B_ALONG>(sh.b[step & 1], line, red, vb[i]);
            }
            __syncthreads();
        }
    }
}

__device__ __forceinline__ uint32_t thread_row(int i) { return (i < 4 ? 0 : 60) + (threadIdx.x >> 4) * 4 + i; }

// ---- G and U of 128 rows and 64 columns, then h, or dG and dU --------------------------------------------------

struct GateArgs {
    FfnProblem p;
    void* grads;          // backward: dG, then dU, each m rows of ld_grad
    uint64_t ld_grad;
    uint32_t x_vectors, wg_vectors, wu_vectors;
};

template <int ACT, bool BACKWARD>
__global__ void __launch_bounds__(kThreads, 2) ffn_simt_gate_kernel(const GateArgs a, const LaunchCtl ctl) {
    __shared__ __align__(16) Shared sh;
    const FfnProblem& p = a.p;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) init_decode_result(p.ws, ctl, p.result_bytes);
    const uint32_t m0 = blockIdx.x * kTile, f0 = blockIdx.y * 64;
    const float* x = static_cast<const float*>(p.x);
    float acc[8][8];
    product<true, true>(
        sh, acc, (p.k + kStep - 1) / kStep,
        [&](uint32_t step, uint32_t g, float v[4]) {
            uint32_t line, red;
            group_of<true>(g, &line, &red);
            const uint32_t row = m0 + line;
            const int64_t c = static_cast<int64_t>(step) * kStep + red;
            load4(x + row * p.ld_x + c, row < p.m ? p.k - c : 0, a.x_vectors, v);
        },
        [&](uint32_t step, uint32_t g, float v[4]) {
            uint32_t line, red;
            group_of<true>(g, &line, &red);
            const uint32_t row = f0 + (line & 63u);
            const int64_t c = static_cast<int64_t>(step) * kStep + red;
            const bool gate = line < 64;
            const float* w = static_cast<const float*>(gate ? p.wg : p.wu) + row * (gate ? p.ld_wg : p.ld_wu) + c;
            load4(w, row < p.f ? p.k - c : 0, gate ? a.wg_vectors : a.wu_vectors, v);
        });
    const uint32_t col = f0 + (threadIdx.x & 15u) * 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t row = m0 + thread_row(i);
        if (row >= p.m || col >= p.f) continue;
        const uint32_t keep = p.drop.threshold ? dropout_keep8(p.drop, row, col >> 3) >> (col & 7u) : 0xfu;
        const uint64_t at = row * p.ld_h + col, to = row * a.ld_grad + col;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (col + j >= p.f) break;
            const float g = acc[i][j], u = acc[i][j + 4];
            if (!BACKWARD) {
                static_cast<float*>(p.h)[at + j] = gated_value<ACT, false>(g, u, (keep >> j) & 1u, p.drop.scale);
            } else {
                float dg, du;
                gated_gradients<ACT, false>(g, u, static_cast<const float*>(p.dh)[at + j], (keep >> j) & 1u, p.drop.scale, &dg, &du);
                static_cast<float*>(a.grads)[to + j] = dg;
                static_cast<float*>(a.grads)[p.m * a.ld_grad + to + j] = du;
            }
        }
    }
}

// ---- dx = [dG dU] [Wg; Wu] --------------------------------------------------------------------------------------

__global__ void __launch_bounds__(kThreads, 2) ffn_simt_dx_kernel(const GateArgs a) {
    __shared__ __align__(16) Shared sh;
    const FfnProblem& p = a.p;
    const uint32_t m0 = blockIdx.x * kTile, c0 = blockIdx.y * kTile;
    const uint32_t half = (p.f + kStep - 1) / kStep;
    const float* grads = static_cast<const float*>(a.grads);
    float acc[8][8];
    product<true, false>(
        sh, acc, 2 * half,
        [&](uint32_t step, uint32_t g, float v[4]) {
            uint32_t line, red;
            group_of<true>(g, &line, &red);
            const bool up = step >= half;
            const uint64_t row = m0 + line;
            const int64_t c = static_cast<int64_t>(up ? step - half : step) * kStep + red;
            load4(grads + (row + (up ? p.m : 0)) * a.ld_grad + c, row < p.m ? p.f - c : 0, true, v);
        },
        [&](uint32_t step, uint32_t g, float v[4]) {
            uint32_t line, red;
            group_of<false>(g, &line, &red);
            const bool up = step >= half;
            const uint64_t row = static_cast<uint64_t>(up ? step - half : step) * kStep + red;
            const int64_t c = c0 + line;
            const float* w = static_cast<const float*>(up ? p.wu : p.wg) + row * (up ? p.ld_wu : p.ld_wg) + c;
            load4(w, row < p.f ? p.k - c : 0, up ? a.wu_vectors : a.wg_vectors, v);
        });
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t row = m0 + thread_row(i), col = c0 + (j < 4 ? 0 : 60) + (threadIdx.x & 15u) * 4 + j;
            if (row < p.m && col < p.k) static_cast<float*>(p.dx)[row * p.ld_dx + col] = acc[i][j];
        }
}

// ---- dWg = dG^T x (blockIdx.z = 0), dWu = dU^T x (1) ------------------------------------------------------------

__global__ void __launch_bounds__(kThreads, 2) ffn_simt_dw_kernel(const GateArgs a) {
    __shared__ __align__(16) Shared sh;
    const FfnProblem& p = a.p;
    const uint32_t f0 = blockIdx.x * kTile, c0 = blockIdx.y * kTile;
    const float* grads = static_cast<const float*>(a.grads) + (blockIdx.z ? p.m * a.ld_grad : 0);
    const float* x = static_cast<const float*>(p.x);
    float acc[8][8];
    product<false, false>(
        sh, acc, (p.m + kStep - 1) / kStep,
        [&](uint32_t step, uint32_t g, float v[4]) {
            uint32_t line, red;
            group_of<false>(g, &line, &red);
            const uint64_t row = static_cast<uint64_t>(step) * kStep + red;
            const int64_t c = f0 + line;
            load4(grads + row * a.ld_grad + c, row < p.m ? p.f - c : 0, true, v);
        },
        [&](uint32_t step, uint32_t g, float v[4]) {
            uint32_t line, red;
            group_of<false>(g, &line, &red);
            const uint64_t row = static_cast<uint64_t>(step) * kStep + red;
            const int64_t c = c0 + line;
            load4(x + row * p.ld_x + c, row < p.m ? p.k - c : 0, a.x_vectors, v);
        });
    float* out = static_cast<float*>(blockIdx.z ? p.dwu : p.dwg);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t row = f0 + thread_row(i), col = c0 + (j < 4 ? 0 : 60) + (threadIdx.x & 15u) * 4 + j;
            if (row < p.f && col < p.k) out[row * p.ld_dw + col] = acc[i][j];
        }
}

uint64_t grad_pitch(uint64_t f) { return (f + 7) & ~7ull; }

GateArgs make_args(const FfnProblem& p) {
    GateArgs a{};
    a.p = p;
    a.grads = reinterpret_cast<uint8_t*>(p.ws) + kFfnWsHeader;
    a.ld_grad = grad_pitch(p.f);
    a.x_vectors = p.ld_x % 4 == 0;
    a.wg_vectors = p.ld_wg % 4 == 0;
    a.wu_vectors = p.ld_wu % 4 == 0;
    return a;
}

uint32_t tiles(uint64_t n, uint32_t t) { return static_cast<uint32_t>((n + t - 1) / t); }

template <bool BACKWARD>
void launch_gate(const GateArgs& a, const LaunchCtl& ctl, cudaStream_t stream) {
    const dim3 grid(tiles(a.p.m, kTile), tiles(a.p.f, 64));
    if (a.p.activation == CDMA_ACT_RELU) ffn_simt_gate_kernel<CDMA_ACT_RELU, BACKWARD><<<grid, kThreads, 0, stream>>>(a, ctl);
    else if (a.p.activation == CDMA_ACT_SILU) ffn_simt_gate_kernel<CDMA_ACT_SILU, BACKWARD><<<grid, kThreads, 0, stream>>>(a, ctl);
    else ffn_simt_gate_kernel<CDMA_ACT_GELU, BACKWARD><<<grid, kThreads, 0, stream>>>(a, ctl);
    count_kernel_launch();
}

}  // namespace

uint64_t ffn_simt_workspace(uint64_t m, uint64_t f, bool backward) {
    return kFfnWsHeader + (backward ? 2 * m * grad_pitch(f) * 4 : 0);
}

cudaError_t launch_ffn_simt(const FfnProblem& p, bool backward, const LaunchCtl& ctl, cudaStream_t stream) {
    const GateArgs a = make_args(p);
    timing_before_launch(stream);
    if (!backward) {
        launch_gate<false>(a, ctl, stream);
    } else {
        launch_gate<true>(a, ctl, stream);
        if (p.dx != nullptr) {
            ffn_simt_dx_kernel<<<dim3(tiles(p.m, kTile), tiles(p.k, kTile)), kThreads, 0, stream>>>(a);
            count_kernel_launch();
        }
        if (p.dwg != nullptr) {
            ffn_simt_dw_kernel<<<dim3(tiles(p.f, kTile), tiles(p.k, kTile), 2), kThreads, 0, stream>>>(a);
            count_kernel_launch();
        }
    }
    timing_after_launch(stream);
    return cudaGetLastError();
}

}  // namespace cdma
