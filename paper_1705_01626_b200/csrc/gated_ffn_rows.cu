// Forward pass of the gated feed-forward block for few rows (a decoding step): bound by the bytes of the weights, so
// the kernel is a stream of the weights through registers, each element read once, without shared memory on the way.
//
// A warp multiplies eight rows of Wg and the same eight of Wu (the 16 rows of a warp-level matrix instruction: a
// thread then holds G and U of the same elements) with 8 * TILES rows of x.  The instruction's reduction order is
// free as long as both operands agree, so a lane simply takes 16 neighbouring bytes of a weight row and the same
// columns of a row of x.  The warps of a block share the reduction, turn by turn; their sums meet in shared memory.
//
// The tcgen05 path would bring 256-row tiles of x, nearly all of them zeros, and hand work to SMs by 32 to 128 hidden
// columns; here a block has 8 columns, so every SM streams.
//
// 4-byte elements are split in two tf32 parts (11 bits each, rounded to nearest) and multiplied as high*high +
// high*low + low*high.  The matrix unit cuts its sums off instead of rounding them, so a sum of a few instructions
// is added to the running one on the ordinary units: without that the loss grows with the reduction's length.
#include "chained_launch.cuh"
#include "gated_ffn.cuh"

namespace cdma {
namespace {

constexpr uint32_t kWarps = 8, kThreads = 32 * kWarps;
constexpr uint32_t kUnroll = 4;      // groups of 64 bytes that a warp has on the way at one time

__device__ __forceinline__ uint4 stream16(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// 16 bytes of a row from element `col` on, zeros past its end.  STREAM: read once.
template <typename T, bool VECTORS, bool STREAM>
__device__ __forceinline__ uint4 take16(const T* row, uint32_t col, uint32_t cols, bool there) {
    constexpr uint32_t kCount = 16 / sizeof(T);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (!there || col >= cols) return v;
    if (VECTORS && col + kCount <= cols) {
        if (STREAM) return stream16(row + col);
        return __ldg(reinterpret_cast<const uint4*>(row + col));
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t i = 0; i < kCount; ++i) {
        if (col + i >= cols) break;
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(__ldg(row + col + i));
        else w[i / 2] |= static_cast<uint32_t>(__ldg(reinterpret_cast<const uint16_t*>(row + col + i))) << (16 * (i & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__device__ __forceinline__ void multiply16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void multiply8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t to_tf32(float v) {
    uint32_t r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(v));
    return r;
}
// High and low part of a float; what is not finite has no low part.
__device__ __forceinline__ void split2(uint32_t bits, uint32_t* high, uint32_t* low) {
    const float v = __uint_as_float(bits);
    *high = to_tf32(v);
    const float rest = v - __uint_as_float(*high);
    *low = fabsf(v) < 3.3e38f ? to_tf32(rest) : 0u;
}

// One lane's 16 bytes of a row of Wg, of Wu and of x: two instructions for 2-byte elements, six for 4-byte ones.
template <typename T>
__device__ __forceinline__ void multiply_group(float (&c)[4], const uint4& g, const uint4& u, const uint4& x) {
    if constexpr (sizeof(T) == 2) {
        multiply16<T>(c, g.x, u.x, g.y, u.y, x.x, x.y);
        multiply16<T>(c, g.z, u.z, g.w, u.w, x.z, x.w);
    } else {
        uint32_t gh[4], gl[4], uh[4], ul[4], xh[4], xl[4];
        split2(g.x, &gh[0], &gl[0]); split2(g.y, &gh[1], &gl[1]); split2(g.z, &gh[2], &gl[2]); split2(g.w, &gh[3], &gl[3]);
        split2(u.x, &uh[0], &ul[0]); split2(u.y, &uh[1], &ul[1]); split2(u.z, &uh[2], &ul[2]); split2(u.w, &uh[3], &ul[3]);
        split2(x.x, &xh[0], &xl[0]); split2(x.y, &xh[1], &xl[1]); split2(x.z, &xh[2], &xl[2]); split2(x.w, &xh[3], &xl[3]);
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            multiply8(c, gl[i], ul[i], gl[i + 1], ul[i + 1], xh[i], xh[i + 1]);
            multiply8(c, gh[i], uh[i], gh[i + 1], uh[i + 1], xl[i], xl[i + 1]);
            multiply8(c, gh[i], uh[i], gh[i + 1], uh[i + 1], xh[i], xh[i + 1]);
        }
    }
}

template <typename T, int TILES, bool VECTORS, int ACT>
__global__ void __launch_bounds__(kThreads) ffn_rows_kernel(const FfnProblem p, const LaunchCtl ctl) {
    constexpr uint32_t kCount = 16 / sizeof(T);         // elements of a lane's 16 bytes
    constexpr uint32_t kGroup = 4 * kCount;             // reduction elements of a group: four lanes' 16 bytes
    __shared__ float sums[kWarps][TILES][4][32];
    const uint32_t warp = threadIdx.x >> 5, lane = lane_id(), row8 = lane >> 2, quad = lane & 3u;
    const uint32_t f0 = blockIdx.x * 8;
    let_next_start();
    wait_for_previous();
    if (blockIdx.x == 0 && threadIdx.x == 0) init_decode_result(p.ws, ctl, p.result_bytes);

    const bool feature = f0 + row8 < p.f;
    const T* wg = static_cast<const T*>(p.wg) + (f0 + row8) * p.ld_wg;
    const T* wu = static_cast<const T*>(p.wu) + (f0 + row8) * p.ld_wu;
    const T* x = static_cast<const T*>(p.x) + row8 * p.ld_x;
    float total[TILES][4];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) total[t][i] = 0.0f;

    // a warp takes kUnroll groups that follow each other, then the next warp, round the block
    for (uint32_t base = warp * kUnroll * kGroup; base < p.k; base += kWarps * kUnroll * kGroup) {
        uint4 g[kUnroll], u[kUnroll];
#pragma unroll
        for (uint32_t i = 0; i < kUnroll; ++i) {
            const uint32_t col = base + i * kGroup + quad * kCount;
            g[i] = take16<T, VECTORS, VECTORS>(wg, col, p.k, feature);
            u[i] = take16<T, VECTORS, VECTORS>(wu, col, p.k, feature);
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (uint32_t i = 0; i < kUnroll; ++i) {
                const uint32_t col = base + i * kGroup + quad * kCount;
                const uint4 v = take16<T, VECTORS, false>(x + 8ull * t * p.ld_x, col, p.k, 8 * t + row8 < p.m);
                multiply_group<T>(c, g[i], u[i], v);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) total[t][i] += c[i];
        }
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[warp][t][i][lane] = total[t][i];
    __syncthreads();

    // Of element (row r of x, hidden column j of the eight) the sums lie in lane 4 j + r / 2 of the row's tile: value
    // r % 2 for G, 2 + r % 2 for U.
    for (uint32_t e = threadIdx.x; e < 64 * TILES; e += kThreads) {
        const uint32_t r = e >> 3, j = e & 7u, tile = r >> 3, at = 4 * j + ((r & 7u) >> 1), odd = r & 1u;
        if (r >= p.m || f0 + j >= p.f) continue;
        float gate = 0.0f, up = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < kWarps; ++w) {
            gate += sums[w][tile][odd][at];
            up += sums[w][tile][2 + odd][at];
        }
        const uint32_t keep = p.drop.threshold ? dropout_keep8(p.drop, r, f0 >> 3) : 0xffu;
        static_cast<T*>(p.h)[r * p.ld_h + f0 + j] =
            from_float<T>(gated_value<ACT, sizeof(T) == 2>(gate, up, (keep >> j) & 1u, p.drop.scale));
    }
}

template <typename T, int TILES, bool VECTORS>
cudaError_t launch_act(const FfnProblem& p, const LaunchCtl& ctl, cudaStream_t stream) {
    const uint32_t grid = (p.f + 7) / 8;
    if (p.activation == CDMA_ACT_RELU) return launch_chained(ffn_rows_kernel<T, TILES, VECTORS, CDMA_ACT_RELU>, grid, kThreads, 0, 0, stream, p, ctl);
    if (p.activation == CDMA_ACT_SILU) return launch_chained(ffn_rows_kernel<T, TILES, VECTORS, CDMA_ACT_SILU>, grid, kThreads, 0, 0, stream, p, ctl);
    return launch_chained(ffn_rows_kernel<T, TILES, VECTORS, CDMA_ACT_GELU>, grid, kThreads, 0, 0, stream, p, ctl);
}
template <bool VECTORS>
cudaError_t launch_tiles(const FfnProblem& p, const LaunchCtl& ctl, cudaStream_t stream) {
    if (p.m <= 8) return launch_act<float, 1, VECTORS>(p, ctl, stream);
    if (p.m <= 16) return launch_act<float, 2, VECTORS>(p, ctl, stream);
    return launch_act<float, 4, VECTORS>(p, ctl, stream);
}

}  // namespace

cudaError_t launch_ffn_rows(const FfnProblem& p, const LaunchCtl& ctl, cudaStream_t stream) {
    timing_before_launch(stream);
    const bool vectors = p.ld_wg % 4 == 0 && p.ld_wu % 4 == 0 && (p.ld_x % 4 == 0 || p.m == 1);
    const cudaError_t e = vectors ? launch_tiles<true>(p, ctl, stream) : launch_tiles<false>(p, ctl, stream);
    timing_after_launch(stream);
    return e;
}

}  // namespace cdma
