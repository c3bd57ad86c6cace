// The gated feed-forward block for 2-byte types on the matrix units (tcgen05): three products with one kernel.
//
//   GATE   G and U of 256 rows and 128 hidden columns: A = x, B = the tile's 128 rows of Wg next to those of Wu, so
//          that an accumulator of 256 columns holds G and U of the same elements and its reader has both at hand.
//          The reader writes h (forward), or dG and dU (backward, after reading dh).
//   DX     256 x 256 of dx: A = dG then dU, B = Wg then Wu, one reduction over both.
//   DW     256 x 256 of dWg or dWu: A = dG^T or dU^T, B = x.
//
// A pair of CTAs on two SMs shares one tile (cta_group::2): each holds half of A's and half of B's rows, and the
// accumulator of its half of the output rows.  In GATE one CTA brings Wg's rows and the other Wu's.  Operands arrive
// by TMA in 128-byte swizzled steps of 64 reduction elements through a ring of six; one thread issues the matrix
// instructions; eight warps read the finished accumulator while the other of two collects the next tile.  Operands
// whose rows, not their reduction, are contiguous in memory (B of DX, both of DW) are taken as they lie, by the
// descriptors' major bits: nothing is transposed.
//
// Sizes that are no multiple of a tile need nothing: TMA fills with zeros outside the matrix and the readers store
// what is inside.  TMA wants 16-byte row strides; an operand with another stride is copied first (pack_kernel).
#include "gated_ffn.cuh"
#include "tcgen05.cuh"
#include "tensor_map.h"

namespace cdma {
namespace {

constexpr uint32_t kStep = 64;                       // reduction elements per step: 128 bytes
constexpr uint32_t kStages = 6;
constexpr uint32_t kOperandBytes = 128 * kStep * 2;  // one CTA's half of A or of B: 128 rows
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr uint32_t kTileRows = 256, kTileCols = 256;
constexpr uint32_t kAccumulators = 2;
constexpr uint32_t kReaderWarps = 8;
constexpr uint32_t kThreads = 32 * (4 + kReaderWarps);
constexpr uint32_t kBand = 16;                       // tile rows that are walked together

enum Mode { kGate = 0, kDx = 1, kDw = 2 };

struct __align__(8) Control {
    uint64_t full[kStages], empty[kStages], done[kAccumulators], free_[kAccumulators];
    uint32_t tmem, gave_up;
};
constexpr uint32_t kSharedBytes = kStages * kStageBytes + sizeof(Control) + 1024;

struct MmaArgs {
    FfnProblem p;
    uint32_t tile_rows, tile_cols;      // tiles of the output (DW: rows of both gradients)
    uint32_t steps;                     // per tile; DX: of each half
    uint32_t parts;                     // DX: 2 halves of the reduction, else 1
    void* grads;                        // dG, then dU: m rows of ld_grad
    uint64_t ld_grad;
    uint32_t backward;
};

// Tiles in bands of kBand tile rows, down a band's column first: the tiles that run at one time then share few rows
// of either operand, which stay in L2.
struct TilePlace {
    uint32_t row, col;
};
__device__ __forceinline__ TilePlace place_of(const MmaArgs& a, uint32_t tile) {
    const uint32_t per_band = kBand * a.tile_cols;
    const uint32_t band = tile / per_band, rest = tile % per_band;
    const uint32_t height = min(kBand, a.tile_rows - band * kBand);
    return {band * kBand + rest % height, rest / height};
}

// Values of 32 neighbouring columns of one row, in pairs; `there` of them exist.
template <typename T>
__device__ __forceinline__ void store_row(T* to, const uint32_t (&pairs)[16], int64_t there) {
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(to));
    if (there >= 32 && (at & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            reinterpret_cast<uint4*>(to)[i] = make_uint4(pairs[4 * i], pairs[4 * i + 1], pairs[4 * i + 2], pairs[4 * i + 3]);
        return;
    }
    uint16_t* words = reinterpret_cast<uint16_t*>(to);
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < there) words[i] = static_cast<uint16_t>(pairs[i >> 1] >> (16 * (i & 1)));
}
template <typename T>
__device__ __forceinline__ void load_row(const T* from, uint32_t (&pairs)[16], int64_t there) {
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(from));
    if (there >= 32 && (at & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(from)[i];
            pairs[4 * i] = v.x; pairs[4 * i + 1] = v.y; pairs[4 * i + 2] = v.z; pairs[4 * i + 3] = v.w;
        }
        return;
    }
    const uint16_t* words = reinterpret_cast<const uint16_t*>(from);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t lo = 2 * i < there ? words[2 * i] : 0, hi = 2 * i + 1 < there ? words[2 * i + 1] : 0;
        pairs[i] = lo | hi << 16;
    }
}

// 32 columns of G and of U: h, or dG and dU.
template <typename T, int ACT>
__device__ __forceinline__ void finish_gate(const MmaArgs& a, uint32_t row, uint32_t col, const uint32_t (&g)[32],
                                            const uint32_t (&u)[32], const uint32_t (&dh)[16]) {
    const FfnProblem& p = a.p;
    uint32_t first[16], second[16];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const uint32_t keep = p.drop.threshold ? dropout_keep8(p.drop, row, (col >> 3) + b) : 0xffu;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const int i = 8 * b + j;
            const float g0 = __uint_as_float(g[i]), g1 = __uint_as_float(g[i + 1]);
            const float u0 = __uint_as_float(u[i]), u1 = __uint_as_float(u[i + 1]);
            const bool k0 = (keep >> j) & 1u, k1 = (keep >> (j + 1)) & 1u;
            if (!a.backward) {
                first[i >> 1] = pack2<T>(gated_value<ACT, true>(g0, u0, k0, p.drop.scale), gated_value<ACT, true>(g1, u1, k1, p.drop.scale));
            } else {
                const float2 e = unpack2<T>(dh[i >> 1]);
                float dg0, du0, dg1, du1;
                gated_gradients<ACT, true>(g0, u0, e.x, k0, p.drop.scale, &dg0, &du0);
                gated_gradients<ACT, true>(g1, u1, e.y, k1, p.drop.scale, &dg1, &du1);
                first[i >> 1] = pack2<T>(dg0, dg1);
                second[i >> 1] = pack2<T>(du0, du1);
            }
        }
    }
    if (row >= p.m || col >= p.f) return;
    if (!a.backward) {
        store_row(static_cast<T*>(p.h) + row * p.ld_h + col, first, static_cast<int64_t>(p.f) - col);
    } else {        // the pitch of dG and dU is a multiple of 64: whole groups fit
        T* to = static_cast<T*>(a.grads) + row * a.ld_grad + col;
        store_row(to, first, 32);
        store_row(to + p.m * a.ld_grad, second, 32);
    }
}

template <int MODE, typename T, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
ffn_mma_kernel(const __grid_constant__ CUtensorMap map_a0, const __grid_constant__ CUtensorMap map_a1,
               const __grid_constant__ CUtensorMap map_b0, const __grid_constant__ CUtensorMap map_b1,
               const __grid_constant__ MmaArgs a, const LaunchCtl ctl) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (shared_address(smem_raw) + 1023u) & ~1023u;
    Control& c = *reinterpret_cast<Control*>(smem_raw + (base - shared_address(smem_raw)) + kStages * kStageBytes);
    const uint32_t warp = threadIdx.x >> 5, lane = lane_id(), rank = cluster_rank();
    const uint32_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t tiles = a.tile_rows * a.tile_cols, steps = a.steps * a.parts;
    constexpr bool kARows = MODE == kDw, kBRows = MODE != kGate;
    constexpr uint32_t kFormat = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1 : 0;

    if (MODE == kGate && blockIdx.x == 0 && threadIdx.x == 0) init_decode_result(a.p.ws, ctl, a.p.result_bytes);
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kStages; ++i) {
            mbar_init(shared_address(&c.full[i]), 1);
            mbar_init(shared_address(&c.empty[i]), 1);
        }
        for (uint32_t i = 0; i < kAccumulators; ++i) {
            mbar_init(shared_address(&c.done[i]), 1);
            mbar_init(shared_address(&c.free_[i]), 2 * kReaderWarps);
        }
        c.gave_up = 0;
        mbar_init_fence();
    }
    if (warp == 2) tmem_alloc_pair(shared_address(&c.tmem), kAccumulators * kTileCols);
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync();
    tcgen05_fence_after();
    const uint32_t tmem = c.tmem;
    volatile uint32_t* gave_up = &c.gave_up;

    if (warp == 0 && lane == 0) {
        // brings this CTA's halves of A and B; the bytes of both CTAs are counted by the first one's barrier
        tma_prefetch_map(&map_a0);
        tma_prefetch_map(&map_b0);
        uint32_t stage = 0, phase = 0;
        bool fine = true;
        for (uint32_t tile = pair; fine && tile < tiles; tile += pairs) {
            const TilePlace at = place_of(a, tile);
            // DW: the upper half of the tile rows are dU's
            const bool second = MODE == kDw && at.row >= a.tile_rows / 2;
            const uint32_t row = (second ? at.row - a.tile_rows / 2 : at.row) * kTileRows + rank * 128;
            const uint32_t col = MODE == kGate ? at.col * 128 : at.col * kTileCols + rank * 128;
            for (uint32_t s = 0; s < steps; ++s) {
                if (!(fine = mbar_wait(shared_address(&c.empty[stage]), phase ^ 1u, gave_up, ctl.wait_limit_ns))) break;
                const uint32_t bar = in_cta(shared_address(&c.full[stage]), 0);
                if (rank == 0) mbar_expect(shared_address(&c.full[stage]), 2 * kStageBytes);
                const uint32_t dst_a = base + stage * kStageBytes, dst_b = dst_a + kOperandBytes;
                const bool up = MODE == kDx && s >= a.steps;
                const uint32_t r = (up ? s - a.steps : s) * kStep;
                const CUtensorMap* ma = (MODE == kDx ? up : second) ? &map_a1 : &map_a0;
                const CUtensorMap* mb = (MODE == kGate ? rank != 0 : up) ? &map_b1 : &map_b0;
                if (kARows) {
                    tma_load_pair(dst_a, ma, row, r, bar);
                    tma_load_pair(dst_a + kOperandBytes / 2, ma, row + 64, r, bar);
                } else {
                    tma_load_pair(dst_a, ma, r, row, bar);
                }
                if (kBRows) {
                    tma_load_pair(dst_b, mb, col, r, bar);
                    tma_load_pair(dst_b + kOperandBytes / 2, mb, col + 64, r, bar);
                } else {
                    tma_load_pair(dst_b, mb, r, col, bar);
                }
                if (++stage == kStages) { stage = 0; phase ^= 1u; }
            }
        }
        // the last steps' releases have arrived here before this CTA's shared memory goes
        for (uint32_t i = 0; fine && i < kStages; ++i) {
            fine = mbar_wait(shared_address(&c.empty[stage]), phase ^ 1u, gave_up, ctl.wait_limit_ns);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        constexpr uint32_t kDesc = mma_desc(kFormat, kARows, kBRows, kTileRows, kTileCols);
        // Reduction-contiguous rows lie 128 bytes apart, 8 rows in 1024; a sub-step of 16 is 32 bytes on.  Else a
        // block of 64 rows is 8192 bytes, 8 reduction lines are 1024, and a sub-step of 16 is 2048 bytes on.
        uint32_t stage = 0, phase = 0, n = 0;
        bool fine = true;
        for (uint32_t tile = pair; fine && tile < tiles; tile += pairs, ++n) {
            const uint32_t acc = n & 1u;
            if (!(fine = mbar_wait(shared_address(&c.free_[acc]), ((n >> 1) & 1u) ^ 1u, gave_up, ctl.wait_limit_ns))) break;
            tcgen05_fence_after();
            for (uint32_t s = 0; s < steps; ++s) {
                if (!(fine = mbar_wait(shared_address(&c.full[stage]), phase, gave_up, ctl.wait_limit_ns))) break;
                tcgen05_fence_after();
                const uint32_t at_a = base + stage * kStageBytes, at_b = at_a + kOperandBytes;
#pragma unroll
                for (uint32_t i = 0; i < kStep / 16; ++i) {
                    const uint64_t da = kARows ? operand_desc(at_a + i * 2048, 8192, 1024) : operand_desc(at_a + i * 32, 16, 1024);
                    const uint64_t db = kBRows ? operand_desc(at_b + i * 2048, 8192, 1024) : operand_desc(at_b + i * 32, 16, 1024);
                    mma_pair(tmem + acc * kTileCols, da, db, kDesc, s != 0 || i != 0);
                }
                mma_commit_pair(shared_address(&c.empty[stage]));
                if (++stage == kStages) { stage = 0; phase ^= 1u; }
            }
            if (fine) mma_commit_pair(shared_address(&c.done[acc]));
        }
    } else if (warp >= 4) {
        const uint32_t quarter = warp & 3u, half = (warp - 4) >> 2;
        uint32_t n = 0;
        for (uint32_t tile = pair; tile < tiles; tile += pairs, ++n) {
            const TilePlace at = place_of(a, tile);
            const uint32_t acc = n & 1u;
            const uint32_t from = tmem + acc * kTileCols + (quarter * 32u << 16);
            const FfnProblem& p = a.p;
            if (MODE == kGate) {
                const uint32_t row = at.row * kTileRows + rank * 128 + quarter * 32 + lane;
                uint32_t dh[16] = {};
                bool fine = true;
#pragma unroll 1
                for (uint32_t i = 0; i < 2; ++i) {
                    const uint32_t within = half * 64 + i * 32, col = at.col * 128 + within;
                    if (a.backward && row < p.m && col < p.f)       // on its way while the accumulator is still collected
                        load_row(static_cast<const T*>(p.dh) + row * p.ld_h + col, dh, static_cast<int64_t>(p.f) - col);
                    if (i == 0) {
                        if (!(fine = mbar_wait(shared_address(&c.done[acc]), (n >> 1) & 1u, gave_up, ctl.wait_limit_ns))) break;
                        tcgen05_fence_after();
                    }
                    __syncwarp();
                    uint32_t g[32], u[32];
                    tmem_load32(from + within, g);
                    tmem_load32(from + 128 + within, u);
                    tmem_load_wait();
                    finish_gate<T, ACT>(a, row, col, g, u, dh);
                }
                if (!fine) break;
            } else {
                if (!mbar_wait(shared_address(&c.done[acc]), (n >> 1) & 1u, gave_up, ctl.wait_limit_ns)) break;
                tcgen05_fence_after();
                const bool second = MODE == kDw && at.row >= a.tile_rows / 2;
                const uint32_t row = (second ? at.row - a.tile_rows / 2 : at.row) * kTileRows + rank * 128 + quarter * 32 + lane;
                T* out = static_cast<T*>(MODE == kDx ? p.dx : second ? p.dwu : p.dwg);
                const uint64_t ld = MODE == kDx ? p.ld_dx : p.ld_dw;
                const uint32_t rows = MODE == kDx ? p.m : p.f;
#pragma unroll 1
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t within = half * 128 + i * 32, col = at.col * kTileCols + within;
                    __syncwarp();
                    uint32_t v[32], packed[16];
                    tmem_load32(from + within, v);
                    tmem_load_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) packed[j] = pack2<T>(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
                    if (row < rows && col < p.k) store_row(out + row * ld + col, packed, static_cast<int64_t>(p.k) - col);
                }
            }
            __syncwarp();
            tcgen05_fence_before();
            if (lane == 0) mbar_arrive_cluster(in_cta(shared_address(&c.free_[acc]), 0));
        }
    }
    __syncwarp();
    __syncthreads();
    if (*gave_up) {
        if (threadIdx.x == 0) report_decode_error(a.p.ws, ctl, CDMA_ERR_TIMEOUT);
        // copies and matrix instructions that are still under way end within microseconds
        for (uint32_t i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 2) tmem_free_pair(tmem, kAccumulators * kTileCols);
}

// ---- operands whose row stride TMA cannot take --------------------------------------------------------------------

struct PackArgs {
    struct One {
        const uint16_t* from;
        uint16_t* to;
        uint64_t ld_from, ld_to;
        uint32_t rows, cols;
    } one[3];
    uint32_t count;
};
__global__ void __launch_bounds__(256) pack_kernel(const PackArgs a) {
    for (uint32_t i = 0; i < a.count; ++i) {
        const PackArgs::One& o = a.one[i];
        for (uint32_t row = blockIdx.x; row < o.rows; row += gridDim.x)
            for (uint32_t col = threadIdx.x; col < o.cols; col += blockDim.x) o.to[row * o.ld_to + col] = o.from[row * o.ld_from + col];
    }
}

uint64_t pitch_of(uint64_t cols) { return (cols + 63) & ~63ull; }
uint64_t round256(uint64_t n) { return (n + 255) & ~255ull; }
bool takes_tma(uint64_t ld) { return ld % 8 == 0; }
uint32_t tiles(uint64_t n, uint32_t t) { return static_cast<uint32_t>((n + t - 1) / t); }

// Everything behind the result words: dG and dU, then copies of operands with odd strides.
struct Layout {
    uint64_t grads, x, wg, wu, end;
};
Layout layout_of(uint64_t m, uint64_t k, uint64_t f, uint64_t ld_x, uint64_t ld_wg, uint64_t ld_wu, bool backward) {
    Layout l;
    l.grads = kFfnWsHeader;
    l.x = l.grads + (backward ? round256(2 * m * pitch_of(f) * 2) : 0);
    l.wg = l.x + (takes_tma(ld_x) ? 0 : round256(m * pitch_of(k) * 2));
    l.wu = l.wg + (takes_tma(ld_wg) ? 0 : round256(f * pitch_of(k) * 2));
    l.end = l.wu + (takes_tma(ld_wu) ? 0 : round256(f * pitch_of(k) * 2));
    return l;
}

struct Matrix {
    const void* p;
    uint64_t rows, cols, ld;
};
// Map of a 2-byte matrix in boxes of 64 columns and `lines` rows.
bool make_map(CUtensorMap* map, const Matrix& m, int dtype, uint32_t lines) {
    return encode_matrix_map(map, dtype == CDMA_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.p,
                             m.rows, m.cols, m.ld, kStep, lines, CU_TENSOR_MAP_SWIZZLE_128B);
}

uint32_t grid_for(uint64_t n_tiles) {
    static const uint32_t sms = [] {
        int dev = 0, n = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) n = 148;
        return static_cast<uint32_t>(n);
    }();
    const uint64_t pairs = sms / 2;
    return 2 * static_cast<uint32_t>(n_tiles < pairs ? n_tiles : pairs);
}

template <int MODE, typename T, int ACT>
cudaError_t launch_mode(const CUtensorMap (&maps)[4], const MmaArgs& a, const LaunchCtl& ctl, cudaStream_t stream) {
    auto kernel = ffn_mma_kernel<MODE, T, ACT>;
    const cudaError_t e = opt_in_shared_memory(reinterpret_cast<const void*>(kernel), kSharedBytes);
    if (e != cudaSuccess) return e;
    kernel<<<grid_for(static_cast<uint64_t>(a.tile_rows) * a.tile_cols), kThreads, kSharedBytes, stream>>>(
        maps[0], maps[1], maps[2], maps[3], a, ctl);
    count_kernel_launch();
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_all(const FfnProblem& p, bool backward, const LaunchCtl& ctl, cudaStream_t stream) {
    const Layout l = layout_of(p.m, p.k, p.f, p.ld_x, p.ld_wg, p.ld_wu, backward);
    uint8_t* ws = reinterpret_cast<uint8_t*>(p.ws);
    Matrix x{p.x, p.m, p.k, p.ld_x}, wg{p.wg, p.f, p.k, p.ld_wg}, wu{p.wu, p.f, p.k, p.ld_wu};
    PackArgs pack{};
    uint64_t rows = 0;
    const uint64_t at[3] = {l.x, l.wg, l.wu};
    Matrix* all[3] = {&x, &wg, &wu};
    for (int i = 0; i < 3; ++i) {
        if (takes_tma(all[i]->ld)) continue;
        Matrix& o = *all[i];
        pack.one[pack.count++] = {static_cast<const uint16_t*>(o.p), reinterpret_cast<uint16_t*>(ws + at[i]), o.ld, pitch_of(o.cols),
                                  static_cast<uint32_t>(o.rows), static_cast<uint32_t>(o.cols)};
        o = Matrix{ws + at[i], o.rows, o.cols, pitch_of(o.cols)};
        if (o.rows > rows) rows = o.rows;
    }
    if (pack.count != 0) {
        pack_kernel<<<static_cast<uint32_t>(rows < 148 * 8 ? rows : 148 * 8), 256, 0, stream>>>(pack);
        count_kernel_launch();
    }

    MmaArgs a{};
    a.p = p;
    a.backward = backward;
    a.grads = ws + l.grads;
    a.ld_grad = pitch_of(p.f);
    const Matrix dg{a.grads, p.m, p.f, a.ld_grad}, du{static_cast<T*>(a.grads) + p.m * a.ld_grad, p.m, p.f, a.ld_grad};
    CUtensorMap maps[4];
    a.tile_rows = tiles(p.m, kTileRows);
    a.tile_cols = tiles(p.f, 128);
    a.steps = tiles(p.k, kStep);
    a.parts = 1;
    if (!make_map(&maps[0], x, p.dtype, 128) || !make_map(&maps[2], wg, p.dtype, 128) || !make_map(&maps[3], wu, p.dtype, 128))
        return cudaErrorInvalidValue;
    maps[1] = maps[0];
    cudaError_t e = p.activation == CDMA_ACT_RELU   ? launch_mode<kGate, T, CDMA_ACT_RELU>(maps, a, ctl, stream)
                    : p.activation == CDMA_ACT_SILU ? launch_mode<kGate, T, CDMA_ACT_SILU>(maps, a, ctl, stream)
                                                    : launch_mode<kGate, T, CDMA_ACT_GELU>(maps, a, ctl, stream);
    if (e != cudaSuccess || !backward) return e;

    if (p.dx != nullptr) {
        a.tile_rows = tiles(p.m, kTileRows);
        a.tile_cols = tiles(p.k, kTileCols);
        a.steps = tiles(p.f, kStep);
        a.parts = 2;
        if (!make_map(&maps[0], dg, p.dtype, 128) || !make_map(&maps[1], du, p.dtype, 128) ||
            !make_map(&maps[2], wg, p.dtype, kStep) || !make_map(&maps[3], wu, p.dtype, kStep))
            return cudaErrorInvalidValue;
        e = launch_mode<kDx, T, 0>(maps, a, ctl, stream);
        if (e != cudaSuccess) return e;
    }
    if (p.dwg != nullptr) {
        a.tile_rows = 2 * tiles(p.f, kTileRows);
        a.tile_cols = tiles(p.k, kTileCols);
        a.steps = tiles(p.m, kStep);
        a.parts = 1;
        if (!make_map(&maps[0], dg, p.dtype, kStep) || !make_map(&maps[1], du, p.dtype, kStep) || !make_map(&maps[2], x, p.dtype, kStep))
            return cudaErrorInvalidValue;
        maps[3] = maps[2];
        e = launch_mode<kDw, T, 0>(maps, a, ctl, stream);
    }
    return e;
}

}  // namespace

uint64_t ffn_mma_workspace(uint64_t m, uint64_t k, uint64_t f, uint64_t ld_x, uint64_t ld_wg, uint64_t ld_wu, bool backward) {
    return layout_of(m, k, f, ld_x, ld_wg, ld_wu, backward).end;
}

cudaError_t launch_ffn_mma(const FfnProblem& p, bool backward, const LaunchCtl& ctl, cudaStream_t stream) {
    timing_before_launch(stream);
    const cudaError_t e = p.dtype == CDMA_F16 ? launch_all<__half>(p, backward, ctl, stream)
                                              : launch_all<__nv_bfloat16>(p, backward, ctl, stream);
    timing_after_launch(stream);
    return e;
}

}  // namespace cdma
