// Forward pass of the gated feed-forward block for few rows of 4-byte elements (a decoding step): bound by the bytes of
// the weights, so the kernel is a stream of the weights through registers, each element read once and multiplied with
// every row of x on the ordinary units, which have room for 16 rows beside the stream.  (The tcgen05 kernels would need
// the weights in bf16 planes, written and read again: four times the bytes.  Warp-level matrix instructions on tf32
// halves were slower than the ordinary units: 108 us against the figures below for one row of 4096 x 10944.)
//
// A warp has two hidden columns: two rows of Wg and the same two of Wu.  Its lanes take neighbouring places of a row,
// four elements each, and keep their sums for all rows of x; the rows of x come from L1.  Four warps share a column's
// reduction turn by turn.  Lanes are summed by shuffles, the four warps through shared memory.
#include "chained_launch.cuh"
#include "gated_ffn.cuh"

namespace cdma {
namespace {

constexpr uint32_t kWarps = 8, kThreads = 32 * kWarps;
constexpr uint32_t kSlices = 4;                                  // warps to a reduction
constexpr uint32_t kTurn = 128;                                  // reduction elements of a warp's turn

// A lane's four elements of the 128 from `base` on: neighbours where rows start on 16 bytes, else every 32nd, so that
// the warp's loads stay contiguous either way.  Zeros past the row's end.
template <bool VECTORS, bool STREAM>
__device__ __forceinline__ float4 take4(const float* row, uint32_t base, uint32_t cols) {
    float v[4];
    if (VECTORS) {
        const uint32_t col = base + 4 * lane_id();
        if (col + 4 <= cols) {
            float4 q;
            if (STREAM)
                asm volatile("ld.global.nc.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "l"(row + col));
            else
                q = __ldg(reinterpret_cast<const float4*>(row + col));
            return q;
        }
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = col + i < cols ? __ldg(row + col + i) : 0.0f;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t col = base + 32 * i + lane_id();
            v[i] = col < cols ? __ldg(row + col) : 0.0f;
        }
    }
    return make_float4(v[0], v[1], v[2], v[3]);
}

template <int ROWS, uint32_t kColumns, bool VECTORS, int ACT>
__global__ void __launch_bounds__(kThreads) ffn_rows_kernel(const FfnProblem p, const LaunchCtl ctl) {
    constexpr uint32_t kPerBlock = kWarps / kSlices * kColumns;      // hidden columns
    __shared__ float sums[kWarps][2 * kColumns][ROWS];
    const uint32_t warp = threadIdx.x >> 5, lane = lane_id(), slice = warp % kSlices;
    const uint32_t f0 = blockIdx.x * kPerBlock + warp / kSlices * kColumns;      // the warp's first hidden column
    let_next_start();
    wait_for_previous();
    if (blockIdx.x == 0 && threadIdx.x == 0) init_decode_result(p.ws, ctl, p.result_bytes);

    const float *x = static_cast<const float*>(p.x), *w[2 * kColumns];
#pragma unroll
    for (uint32_t i = 0; i < kColumns; ++i) {       // a column past the last one repeats it
        const uint64_t f = min(f0 + i, p.f - 1);
        w[2 * i] = static_cast<const float*>(p.wg) + f * p.ld_wg;
        w[2 * i + 1] = static_cast<const float*>(p.wu) + f * p.ld_wu;
    }
    float sum[2 * kColumns][ROWS];
#pragma unroll
    for (uint32_t i = 0; i < 2 * kColumns; ++i)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) sum[i][r] = 0.0f;

#pragma unroll (ROWS <= 4 ? 2 : 1)
    for (uint32_t base = slice * kTurn; base < p.k; base += kSlices * kTurn) {
        float4 q[2 * kColumns];
#pragma unroll
        for (uint32_t i = 0; i < 2 * kColumns; ++i) q[i] = take4<VECTORS, VECTORS>(w[i], base, p.k);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float4 v = take4<VECTORS, false>(x + min(static_cast<uint32_t>(r), p.m - 1) * p.ld_x, base, p.k);
#pragma unroll
            for (uint32_t i = 0; i < 2 * kColumns; ++i)
                sum[i][r] = fmaf(q[i].w, v.w, fmaf(q[i].z, v.z, fmaf(q[i].y, v.y, fmaf(q[i].x, v.x, sum[i][r]))));
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < 2 * kColumns; ++i)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float v = sum[i][r];
#pragma unroll
            for (uint32_t d = 16; d != 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
            if (lane == 0) sums[warp][i][r] = v;
        }
    __syncthreads();

    for (uint32_t e = threadIdx.x; e < kPerBlock * ROWS; e += kThreads) {
        const uint32_t r = e / kPerBlock, j = e % kPerBlock, f = blockIdx.x * kPerBlock + j;
        if (r >= p.m || f >= p.f) continue;
        float g = 0.0f, u = 0.0f;
#pragma unroll
        for (uint32_t s = 0; s < kSlices; ++s) {
            g += sums[j / kColumns * kSlices + s][2 * (j % kColumns)][r];
            u += sums[j / kColumns * kSlices + s][2 * (j % kColumns) + 1][r];
        }
        const uint32_t keep = p.drop.threshold ? dropout_keep8(p.drop, r, f >> 3) >> (f & 7u) : 1u;
        static_cast<float*>(p.h)[r * p.ld_h + f] = gated_value<ACT, false>(g, u, keep & 1u, p.drop.scale);
    }
}

template <int ROWS, uint32_t COLUMNS, bool VECTORS>
cudaError_t launch_act(const FfnProblem& p, const LaunchCtl& ctl, cudaStream_t stream) {
    constexpr uint32_t kPerBlock = kWarps / kSlices * COLUMNS;
    const uint32_t grid = (p.f + kPerBlock - 1) / kPerBlock;
    if (p.activation == CDMA_ACT_RELU) return launch_chained(ffn_rows_kernel<ROWS, COLUMNS, VECTORS, CDMA_ACT_RELU>, grid, kThreads, 0, 0, stream, p, ctl);
    if (p.activation == CDMA_ACT_SILU) return launch_chained(ffn_rows_kernel<ROWS, COLUMNS, VECTORS, CDMA_ACT_SILU>, grid, kThreads, 0, 0, stream, p, ctl);
    return launch_chained(ffn_rows_kernel<ROWS, COLUMNS, VECTORS, CDMA_ACT_GELU>, grid, kThreads, 0, 0, stream, p, ctl);
}
template <bool VECTORS>
cudaError_t launch_rows(const FfnProblem& p, const LaunchCtl& ctl, cudaStream_t stream) {
    if (p.m == 1) return launch_act<1, 2, VECTORS>(p, ctl, stream);
    if (p.m == 2) return launch_act<2, 2, VECTORS>(p, ctl, stream);
    if (p.m <= 4) return launch_act<4, 2, VECTORS>(p, ctl, stream);
    if (p.m <= 8) return launch_act<8, 4, VECTORS>(p, ctl, stream);
    return launch_act<16, 2, VECTORS>(p, ctl, stream);
}

}  // namespace

cudaError_t launch_ffn_rows(const FfnProblem& p, const LaunchCtl& ctl, cudaStream_t stream) {
    timing_before_launch(stream);
    const bool vectors = p.ld_wg % 4 == 0 && p.ld_wu % 4 == 0 && (p.ld_x % 4 == 0 || p.m == 1);
    const cudaError_t e = vectors ? launch_rows<true>(p, ctl, stream) : launch_rows<false>(p, ctl, stream);
    timing_after_launch(stream);
    return e;
}

}  // namespace cdma
