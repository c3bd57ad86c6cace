// The gated feed-forward block on the matrix units (tcgen05).
//
//   gate kernel      G and U of 256 rows and up to 128 hidden columns: A = x, B = the tile's rows of Wg next to those
//                    of Wu, so that an accumulator holds G and U of the same elements and its reader has both at hand.
//                    The reader writes h (forward), or dG and dU (backward, after reading dh).
//   products kernel  256 x 256 tiles of dx (A = dG then dU, B = Wg then Wu, one reduction over both) and of dWg and
//                    dWu (A = dG^T or dU^T, B = x), in one launch: both only need dG and dU.
//
// A pair of CTAs on two SMs shares one tile (cta_group::2): each holds half of A's and half of B's rows, and the
// accumulator of its half of the output rows.  In the gate kernel one CTA brings Wg's rows and the other Wu's.
// Operands arrive by TMA in 128-byte swizzled steps of 64 reduction elements through a ring; one thread issues the
// matrix instructions; eight warps read the finished accumulator while the other of two collects the next tile.
// Operands whose rows, not their reduction, are contiguous in memory (B of dx, both of dW) are taken as they lie, by
// the descriptors' major bits: nothing is transposed.
//
// Sizes that are no multiple of a tile need nothing: TMA fills with zeros outside the matrix and the readers store
// what is inside.  TMA wants 16-byte row strides; an operand with another stride is copied first (prepare_kernel).
//
// 4-byte elements: each operand is split into three bf16 planes (x = high + middle + low, 8 bits each: all 24), and
// the six products of planes that reach 2^-24 of the whole are six parts of one long reduction, the small ones first.
// Six bf16 products cost less than half of what the same sum takes on the ordinary units.
#include "gated_ffn.cuh"
#include "gated_ffn_maps.cuh"
#include "tcgen05.cuh"

namespace cdma {
namespace {

constexpr uint32_t kPairs = 74;                      // pairs of SMs
constexpr uint32_t kStep = 64;                       // reduction elements per step: 128 bytes
constexpr uint32_t kHalfBytes = 128 * kStep * 2;     // one CTA's half of A: 128 rows
constexpr uint32_t kTileRows = 256;
constexpr uint32_t kReaderWarps = 8;
constexpr uint32_t kThreads = 32 * (4 + kReaderWarps);
constexpr uint32_t kBand = 16;                       // tile rows that are walked together
constexpr uint32_t kMaxStages = 9;

template <typename T> struct Planes { static constexpr uint32_t count = 1, products = 1; };
template <> struct Planes<float> { static constexpr uint32_t count = 3, products = 6; };
// Planes of A and of B in the parts of the reduction (4 bits each, the first part lowest).
constexpr uint32_t kPlaneOfA = 0x010120u, kPlaneOfB = 0x001102u;

// Warp-private block of shared memory through which 32 x 32 elements turn: a thread has a row of them in registers,
// memory wants neighbouring threads on neighbouring columns.  Rows are padded by 16 bytes: no bank conflicts.
template <typename T> constexpr uint32_t kTurnPitch = 32 * sizeof(T) + 16;
template <typename T> constexpr uint32_t kTurnBytes = kReaderWarps * 32 * kTurnPitch<T>;

struct __align__(8) Control {
    uint64_t full[kMaxStages], empty[kMaxStages], done[2], free_[2];
    uint32_t tmem, gave_up;
};
template <uint32_t COLS> constexpr uint32_t kStageBytes = kHalfBytes + COLS / 2 * kStep * 2;
// as many steps as fit beside the turning blocks and the barriers (227 KB)
template <typename T, uint32_t COLS> constexpr uint32_t kStagesThatFit =
    (232448 - 1024 - sizeof(Control) - kTurnBytes<T>) / kStageBytes<COLS>;
template <typename T, uint32_t COLS> constexpr uint32_t kStages =
    kStagesThatFit<T, COLS> < kMaxStages ? kStagesThatFit<T, COLS> : kMaxStages;
template <typename T, uint32_t COLS> constexpr uint32_t kSharedBytes =
    1024 + kStages<T, COLS> * kStageBytes<COLS> + kTurnBytes<T> + sizeof(Control);

struct Gradients {      // dG then dU, each in its planes: `m` rows of `ld` 2-byte elements per plane
    uint16_t* at;
    uint64_t ld;
};
struct GateArgs {
    FfnProblem p;
    uint32_t tile_rows, tile_cols, steps, backward;
    Gradients grads;
};
// Tiles of one product.  With splits > 1 each tile's reduction is cut into that many items, which leave sums in 32
// bits for the joining kernel: where there are fewer tiles than pairs of SMs.
struct Product {
    uint32_t tile_rows, tile_cols, steps, parts, splits;
    float* partial;
    uint64_t ld_partial, rows_partial;
};
struct ProductsArgs {
    FfnProblem p;
    Product dx, dw;
};

// What a pair of CTAs does at one time: an output tile and a range of its reduction.
struct Item {
    bool dw, second;          // products: dW; of dWu
    uint32_t row, col;        // of the tile
    uint32_t first, last;     // steps, counted through the parts
    uint32_t steps, split;
};

// Tiles in bands of kBand tile rows, down a band's column first: the tiles that run at one time then share few rows
// of either operand, which stay in L2.
__device__ __forceinline__ void place(uint32_t tile, uint32_t tile_rows, uint32_t tile_cols, uint32_t* row, uint32_t* col) {
    const uint32_t per_band = kBand * tile_cols;
    const uint32_t band = tile / per_band, rest = tile % per_band;
    const uint32_t height = min(kBand, tile_rows - band * kBand);
    *row = band * kBand + rest % height;
    *col = rest / height;
}

template <typename T>
__device__ __forceinline__ uint32_t items_of(const GateArgs& a) { return a.tile_rows * a.tile_cols; }
template <typename T>
__device__ __forceinline__ Item item_of(const GateArgs& a, uint32_t index) {
    Item it{};
    place(index, a.tile_rows, a.tile_cols, &it.row, &it.col);
    it.steps = a.steps;
    it.last = a.steps * Planes<T>::products;
    return it;
}
__device__ __forceinline__ uint32_t items_of(const Product& q) { return q.tile_rows * q.tile_cols * q.splits; }
template <typename T>
__device__ __forceinline__ uint32_t items_of(const ProductsArgs& a) { return items_of(a.dx) + items_of(a.dw); }
template <typename T>
__device__ __forceinline__ Item item_of(const ProductsArgs& a, uint32_t index) {
    Item it{};
    it.dw = index >= items_of(a.dx);
    const Product& q = it.dw ? a.dw : a.dx;
    const uint32_t i = it.dw ? index - items_of(a.dx) : index, tiles = q.tile_rows * q.tile_cols;
    it.split = i / tiles;
    place(i % tiles, q.tile_rows, q.tile_cols, &it.row, &it.col);
    const uint64_t total = static_cast<uint64_t>(q.steps) * q.parts;
    it.first = static_cast<uint32_t>(total * it.split / q.splits);
    it.last = static_cast<uint32_t>(total * (it.split + 1) / q.splits);
    it.steps = q.steps;
    if (it.dw && it.row >= q.tile_rows / 2) {      // the upper half of the tile rows are dWu's
        it.second = true;
        it.row -= q.tile_rows / 2;
    }
    return it;
}

// ---- between registers and memory --------------------------------------------------------------------------------

// Stores the warp's 32 x 32 block: `words` is the thread's row of it (2-byte elements in pairs), `out` its first
// element, `rows` and `cols` what of it exists.
template <typename T, int WORDS>
__device__ __forceinline__ void store_block(uint8_t* turn, const uint32_t (&words)[WORDS], T* out, uint64_t ld, int64_t rows, int64_t cols) {
    static_assert(WORDS * 4 == 32 * sizeof(T), "a row of 32 elements");
    constexpr uint32_t kPitch = kTurnPitch<T>, kVectors = WORDS / 4, kRowsAtOnce = 32 / kVectors;
    const uint32_t lane = lane_id();
    __syncwarp();
#pragma unroll
    for (uint32_t i = 0; i < kVectors; ++i)
        *reinterpret_cast<uint4*>(turn + lane * kPitch + 16 * i) = make_uint4(words[4 * i], words[4 * i + 1], words[4 * i + 2], words[4 * i + 3]);
    __syncwarp();
    if (cols >= 32 && ((reinterpret_cast<uintptr_t>(out) | ld * sizeof(T)) & 15u) == 0) {
        const uint32_t first = lane / kVectors, vector = lane % kVectors;
#pragma unroll
        for (uint32_t i = 0; i < kVectors; ++i) {
            const uint32_t r = i * kRowsAtOnce + first;
            if (r < rows)
                *reinterpret_cast<uint4*>(out + r * ld + vector * (16 / sizeof(T))) = *reinterpret_cast<const uint4*>(turn + r * kPitch + 16 * vector);
        }
    } else if (lane < cols) {
#pragma unroll 8
        for (uint32_t r = 0; r < 32; ++r)
            if (r < rows) out[r * ld + lane] = *reinterpret_cast<const T*>(turn + r * kPitch + lane * sizeof(T));
    }
}
// The other way: the thread's row of a 32 x 32 block, zero where nothing is.
template <typename T, int WORDS>
__device__ __forceinline__ void load_block(uint8_t* turn, uint32_t (&words)[WORDS], const T* in, uint64_t ld, int64_t rows, int64_t cols) {
    constexpr uint32_t kPitch = kTurnPitch<T>, kVectors = WORDS / 4;
    const uint32_t lane = lane_id();
    if (cols >= 32 && ((reinterpret_cast<uintptr_t>(in) | ld * sizeof(T)) & 15u) == 0) {
#pragma unroll
        for (uint32_t i = 0; i < kVectors; ++i) {
            const uint4 v = lane < rows ? reinterpret_cast<const uint4*>(in + lane * ld)[i] : make_uint4(0, 0, 0, 0);
            words[4 * i] = v.x; words[4 * i + 1] = v.y; words[4 * i + 2] = v.z; words[4 * i + 3] = v.w;
        }
        return;
    }
    __syncwarp();
#pragma unroll 8
    for (uint32_t r = 0; r < 32; ++r)
        *reinterpret_cast<T*>(turn + r * kPitch + lane * sizeof(T)) = r < rows && lane < cols ? in[r * ld + lane] : from_float<T>(0.0f);
    __syncwarp();
#pragma unroll
    for (uint32_t i = 0; i < kVectors; ++i) {
        const uint4 v = *reinterpret_cast<const uint4*>(turn + lane * kPitch + 16 * i);
        words[4 * i] = v.x; words[4 * i + 1] = v.y; words[4 * i + 2] = v.z; words[4 * i + 3] = v.w;
    }
}

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

template <typename T> struct RowWords { static constexpr int count = 32 * sizeof(T) / 4; };

template <typename T>
__device__ __forceinline__ void pack_row(const float (&v)[32], uint32_t (&words)[RowWords<T>::count]) {
#pragma unroll
    for (int i = 0; i < 32; i += 4 / sizeof(T)) {
        if constexpr (sizeof(T) == 4) words[i] = __float_as_uint(v[i]);
        else words[i / 2] = pack2<T>(v[i], v[i + 1]);
    }
}
template <typename T>
__device__ __forceinline__ float element(const uint32_t (&words)[RowWords<T>::count], int i) {
    if constexpr (sizeof(T) == 4) {
        return __uint_as_float(words[i]);
    } else {
        const float2 v = unpack2<T>(words[i >> 1]);
        return i & 1 ? v.y : v.x;
    }
}

// One gradient (which: 0 dG, 1 dU) into its planes of the workspace.  The pitch there is a multiple of 64 elements,
// so a block of 32 columns always fits.
template <typename T>
__device__ __forceinline__ void store_gradient(uint8_t* turn, const float (&v)[32], const Gradients& g, uint32_t m, uint32_t which,
                                               uint32_t row, uint32_t col) {
    const int64_t rows = static_cast<int64_t>(m) - row;
    uint16_t* to = g.at + (static_cast<uint64_t>(which) * Planes<T>::count * m + row) * g.ld + col;
    if constexpr (sizeof(T) == 2) {
        uint32_t words[16];
        pack_row<T>(v, words);
        store_block<T>(turn, words, reinterpret_cast<T*>(to), g.ld, rows, 32);
    } else {
        uint32_t words[3][16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            uint32_t lo[3], hi[3];
            split3(v[i], lo);
            split3(v[i + 1], hi);
#pragma unroll
            for (int j = 0; j < 3; ++j) words[j][i / 2] = lo[j] | hi[j] << 16;
        }
#pragma unroll
        for (int j = 0; j < 3; ++j)
            store_block<__nv_bfloat16>(turn, words[j], reinterpret_cast<__nv_bfloat16*>(to + static_cast<uint64_t>(j) * m * g.ld), g.ld, rows, 32);
    }
}

// 32 columns of G and of U of the thread's row (the warp's first row is `row`): h, or dG and dU.
template <typename T, int ACT>
__device__ __forceinline__ void finish_gate(const GateArgs& a, uint8_t* turn, uint32_t row, uint32_t col, const uint32_t (&g)[32],
                                            const uint32_t (&u)[32], const uint32_t (&dh)[RowWords<T>::count]) {
    const FfnProblem& p = a.p;
    constexpr bool kFast = sizeof(T) == 2;
    float first[32], second[32];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const uint32_t keep = p.drop.threshold ? dropout_keep8(p.drop, row + lane_id(), (col >> 3) + b) : 0xffu;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = 8 * b + j;
            const float gv = __uint_as_float(g[i]), uv = __uint_as_float(u[i]);
            const bool kept = (keep >> j) & 1u;
            if (!a.backward) first[i] = gated_value<ACT, kFast>(gv, uv, kept, p.drop.scale);
            else gated_gradients<ACT, kFast>(gv, uv, element<T>(dh, i), kept, p.drop.scale, &first[i], &second[i]);
        }
    }
    if (row >= p.m || col >= p.f) return;       // the same for the whole warp
    if (!a.backward) {
        uint32_t words[RowWords<T>::count];
        pack_row<T>(first, words);
        store_block<T>(turn, words, static_cast<T*>(p.h) + row * p.ld_h + col, p.ld_h, static_cast<int64_t>(p.m) - row, static_cast<int64_t>(p.f) - col);
    } else {
        store_gradient<T>(turn, first, a.grads, p.m, 0, row, col);
        store_gradient<T>(turn, second, a.grads, p.m, 1, row, col);
    }
}

// ---- the three roles of a CTA --------------------------------------------------------------------------------------

template <bool GATE, uint32_t COLS, typename T>
struct Ring {
    static constexpr uint32_t kDepth = kStages<T, COLS>;
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void next() {
        if (++stage == kDepth) { stage = 0; phase ^= 1u; }
    }
};

// One thread per CTA: brings this CTA's halves of A and B; the bytes of both CTAs are counted by the first one's barrier.
template <bool GATE, uint32_t COLS, typename T, typename Args>
__device__ __forceinline__ void run_loader(const Args& a, const CUtensorMap* map_x, const CUtensorMap* map_g, const CUtensorMap* map_wg,
                                           const CUtensorMap* map_wu, uint32_t base, Control& c, const LaunchCtl& ctl) {
    const uint32_t rank = cluster_rank(), items = items_of<T>(a);
    Ring<GATE, COLS, T> ring;
    bool fine = true;
    for (uint32_t index = blockIdx.x >> 1; fine && index < items; index += gridDim.x >> 1) {
        const Item it = item_of<T>(a, index);
        const uint32_t row = it.row * kTileRows + rank * 128;
        const uint32_t col = GATE ? it.col * (COLS / 2) : it.col * COLS + rank * (COLS / 2);
        uint32_t part = it.first / it.steps, r = it.first % it.steps * kStep;
        for (uint32_t s = it.first; s < it.last; ++s) {
            if (!(fine = mbar_wait(shared_address(&c.empty[ring.stage]), ring.phase ^ 1u, &c.gave_up, ctl.wait_limit_ns))) break;
            const uint32_t bar = in_cta(shared_address(&c.full[ring.stage]), 0);
            if (rank == 0) mbar_expect(shared_address(&c.full[ring.stage]), 2 * kStageBytes<COLS>);
            const uint32_t dst_a = base + ring.stage * kStageBytes<COLS>, dst_b = dst_a + kHalfBytes;
            // the products of planes are the outer parts; dx has a half for G and one for U in each
            const bool up = !GATE && !it.dw && (part & 1u);
            const uint32_t product = !GATE && !it.dw ? part >> 1 : part;
            const uint32_t plane_a = sizeof(T) == 4 ? kPlaneOfA >> (4 * product) & 15u : 0;
            const uint32_t plane_b = sizeof(T) == 4 ? kPlaneOfB >> (4 * product) & 15u : 0;
            const uint32_t of_g = (it.dw ? it.second : up) ? Planes<T>::count : 0;
            if constexpr (GATE) {
                tma_load_pair(dst_a, map_x, r, row, plane_a, bar);
                tma_load_pair(dst_b, rank != 0 ? map_wu : map_wg, r, col, plane_b, bar);
            } else if (!it.dw) {
                tma_load_pair(dst_a, map_g, r, row, of_g + plane_a, bar);
                tma_load_pair(dst_a + kHalfBytes / 2, map_g, r, row + 64, of_g + plane_a, bar);
                const CUtensorMap* w = up ? map_wu : map_wg;
#pragma unroll
                for (uint32_t i = 0; i < COLS / 128; ++i) tma_load_pair(dst_b + i * 8192, w, col + 64 * i, r, plane_b, bar);
            } else {
                tma_load_pair(dst_a, map_g, row, r, of_g + plane_a, bar);
                tma_load_pair(dst_a + kHalfBytes / 2, map_g, row + 64, r, of_g + plane_a, bar);
#pragma unroll
                for (uint32_t i = 0; i < COLS / 128; ++i) tma_load_pair(dst_b + i * 8192, map_x, col + 64 * i, r, plane_b, bar);
            }
            ring.next();
            r += kStep;
            if (r >= it.steps * kStep) { r = 0; ++part; }
        }
    }
    // the last steps' releases have arrived here before this CTA's shared memory goes
    for (uint32_t i = 0; fine && i < ring.kDepth; ++i) {
        fine = mbar_wait(shared_address(&c.empty[ring.stage]), ring.phase ^ 1u, &c.gave_up, ctl.wait_limit_ns);
        ring.next();
    }
}

// One thread of the pair: issues the matrix instructions.  A reduction-contiguous operand's rows lie 128 bytes apart,
// eight rows in 1024 bytes, and a sub-step of 16 is 32 bytes on; of the other kind a block of 64 rows is 8192 bytes,
// eight reduction lines are 1024, and a sub-step is 2048 bytes on.
template <bool GATE, uint32_t COLS, typename T, typename Args>
__device__ __forceinline__ void run_issuer(const Args& a, uint32_t base, Control& c, const LaunchCtl& ctl) {
    constexpr uint32_t kFormat = std::is_same<T, __half>::value ? 0 : 1;
    constexpr uint32_t kDesc = mma_desc(kFormat, false, !GATE, kTileRows, COLS);
    constexpr uint32_t kDescDw = mma_desc(kFormat, true, true, kTileRows, COLS);
    const uint32_t items = items_of<T>(a);
    Ring<GATE, COLS, T> ring;
    uint32_t n = 0;
    bool fine = true;
    for (uint32_t index = blockIdx.x >> 1; fine && index < items; index += gridDim.x >> 1, ++n) {
        const Item it = item_of<T>(a, index);
        const uint32_t acc = n & 1u, tmem = c.tmem + acc * COLS;
        const bool a_rows = !GATE && it.dw;
        const uint32_t desc = a_rows ? kDescDw : kDesc;
        const uint64_t like_a = a_rows ? operand_desc(0, 8192, 1024) : operand_desc(0, 16, 1024);
        const uint64_t like_b = GATE ? operand_desc(0, 16, 1024) : operand_desc(0, 8192, 1024);
        const uint32_t step_a = a_rows ? 2048 >> 4 : 32 >> 4;
        constexpr uint32_t step_b = GATE ? 32 >> 4 : 2048 >> 4;
        if (!(fine = mbar_wait(shared_address(&c.free_[acc]), ((n >> 1) & 1u) ^ 1u, &c.gave_up, ctl.wait_limit_ns))) break;
        tcgen05_fence_after();
        for (uint32_t s = it.first; s < it.last; ++s) {
            if (!(fine = mbar_wait(shared_address(&c.full[ring.stage]), ring.phase, &c.gave_up, ctl.wait_limit_ns))) break;
            tcgen05_fence_after();
            const uint32_t at = (base + ring.stage * kStageBytes<COLS>) >> 4;
#pragma unroll
            for (uint32_t i = 0; i < kStep / 16; ++i)
                mma_pair(tmem, like_a + at + i * step_a, like_b + at + (kHalfBytes >> 4) + i * step_b, desc, s != it.first || i != 0);
            mma_commit_pair(shared_address(&c.empty[ring.stage]));
            ring.next();
        }
        if (fine) mma_commit_pair(shared_address(&c.done[acc]));
    }
}

// Eight warps: quarters of the accumulator's rows, every other block of 32 columns.
template <bool GATE, uint32_t COLS, typename T, int ACT, typename Args>
__device__ __forceinline__ void run_readers(const Args& a, uint8_t* turns, Control& c, const LaunchCtl& ctl) {
    const uint32_t warp = (threadIdx.x >> 5) - 4, quarter = warp & 3u, half = warp >> 2, rank = cluster_rank(), lane = lane_id();
    uint8_t* turn = turns + warp * 32 * kTurnPitch<T>;
    const uint32_t items = items_of<T>(a);
    const FfnProblem& p = a.p;
    uint32_t n = 0;
    for (uint32_t index = blockIdx.x >> 1; index < items; index += gridDim.x >> 1, ++n) {
        const Item it = item_of<T>(a, index);
        const uint32_t acc = n & 1u, from = c.tmem + acc * COLS + (quarter * 32u << 16);
        const uint32_t row = it.row * kTileRows + rank * 128 + quarter * 32;      // the warp's first
        const uint32_t done = shared_address(&c.done[acc]), parity = (n >> 1) & 1u;
        bool fine = true;
        if constexpr (GATE) {
            uint32_t dh[RowWords<T>::count] = {};
#pragma unroll 1
            for (uint32_t i = half; i < COLS / 64; i += 2) {
                const uint32_t col = it.col * (COLS / 2) + i * 32;
                if (a.backward && row < p.m && col < p.f)       // on its way while the accumulator is still collected
                    load_block<T>(turn, dh, static_cast<const T*>(p.dh) + row * p.ld_h + col, p.ld_h, static_cast<int64_t>(p.m) - row,
                                  static_cast<int64_t>(p.f) - col);
                if (i == half) {
                    if (!(fine = mbar_wait(done, parity, &c.gave_up, ctl.wait_limit_ns))) break;
                    tcgen05_fence_after();
                }
                __syncwarp();
                uint32_t g[32], u[32];
                tmem_load32(from + i * 32, g);
                tmem_load32(from + COLS / 2 + i * 32, u);
                tmem_load_wait();
                finish_gate<T, ACT>(a, turn, row, col, g, u, dh);
            }
            if (COLS / 64 <= half) fine = mbar_wait(done, parity, &c.gave_up, ctl.wait_limit_ns);
        } else {
            if (!(fine = mbar_wait(done, parity, &c.gave_up, ctl.wait_limit_ns))) break;
            tcgen05_fence_after();
            const Product& q = it.dw ? a.dw : a.dx;
            T* out = static_cast<T*>(!it.dw ? p.dx : it.second ? p.dwu : p.dwg);
            const uint64_t ld = it.dw ? p.ld_dw : p.ld_dx;
            const uint32_t rows = it.dw ? p.f : p.m;
#pragma unroll 1
            for (uint32_t i = half; i < COLS / 32; i += 2) {
                const uint32_t col = it.col * COLS + i * 32;
                __syncwarp();
                uint32_t v[32];
                tmem_load32(from + i * 32, v);
                tmem_load_wait();
                if (row >= rows || col >= p.k) continue;
                if (q.splits > 1) {
                    if (row + lane < rows) {
                        float* to = q.partial + (it.split * q.rows_partial + (it.second ? rows : 0) + row + lane) * q.ld_partial + col;
#pragma unroll
                        for (int j = 0; j < 8; ++j) reinterpret_cast<uint4*>(to)[j] = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                    }
                } else {
                    float values[32];
                    uint32_t words[RowWords<T>::count];
#pragma unroll
                    for (int j = 0; j < 32; ++j) values[j] = __uint_as_float(v[j]);
                    pack_row<T>(values, words);
                    store_block<T>(turn, words, out + row * ld + col, ld, static_cast<int64_t>(rows) - row, static_cast<int64_t>(p.k) - col);
                }
            }
        }
        if (!fine) break;
        __syncwarp();
        tcgen05_fence_before();
        if (lane == 0) mbar_arrive_cluster(in_cta(shared_address(&c.free_[acc]), 0));
    }
}

template <bool GATE, uint32_t COLS, typename T, int ACT, typename Args>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
ffn_mma_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_g,
               const __grid_constant__ CUtensorMap map_wg, const __grid_constant__ CUtensorMap map_wu,
               const __grid_constant__ Args a, const LaunchCtl ctl) {
    extern __shared__ uint8_t smem_raw[];
    constexpr uint32_t kDepth = kStages<T, COLS>;
    const uint32_t raw = shared_address(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* turns = smem_raw + (base - raw) + kDepth * kStageBytes<COLS>;
    Control& c = *reinterpret_cast<Control*>(turns + kTurnBytes<T>);
    const uint32_t warp = threadIdx.x >> 5, lane = lane_id();

    if (GATE && blockIdx.x == 0 && threadIdx.x == 0) init_decode_result(a.p.ws, ctl, a.p.result_bytes);
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kDepth; ++i) {
            mbar_init(shared_address(&c.full[i]), 1);
            mbar_init(shared_address(&c.empty[i]), 1);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            mbar_init(shared_address(&c.done[i]), 1);
            mbar_init(shared_address(&c.free_[i]), 2 * kReaderWarps);
        }
        c.gave_up = 0;
        mbar_init_fence();
    }
    if (warp == 2) tmem_alloc_pair(shared_address(&c.tmem), 2 * COLS);
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync();
    tcgen05_fence_after();

    if (warp == 0 && lane == 0) run_loader<GATE, COLS, T>(a, &map_x, &map_g, &map_wg, &map_wu, base, c, ctl);
    else if (warp == 1 && lane == 0 && cluster_rank() == 0) run_issuer<GATE, COLS, T>(a, base, c, ctl);
    else if (warp >= 4) run_readers<GATE, COLS, T, ACT>(a, turns, c, ctl);

    __syncwarp();
    __syncthreads();
    if (*static_cast<volatile uint32_t*>(&c.gave_up)) {
        if (threadIdx.x == 0) report_decode_error(a.p.ws, ctl, CDMA_ERR_TIMEOUT);
        // copies and matrix instructions that are still under way end within microseconds
        for (uint32_t i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 2) tmem_free_pair(c.tmem, 2 * COLS);
}

// ---- operands that TMA or the matrix units cannot take as they are -------------------------------------------------

// Copies of up to three operands: 2-byte elements with a row stride that is a multiple of 64 elements, or the planes
// of 4-byte elements.  A thread makes eight neighbouring elements.
struct PrepareArgs {
    struct One {
        const void* from;
        uint16_t* to;
        uint64_t ld_from, ld_to, plane;
        uint32_t rows, cols, groups, vectors;      // groups of eight per row
    } one[3];
    uint64_t first[4];      // numbers of the operands' first groups, then the end
};
template <typename T>
__global__ void __launch_bounds__(256) prepare_kernel(const PrepareArgs a) {
    const uint64_t n = blockIdx.x * 256ull + threadIdx.x;
    if (n >= a.first[3]) return;
    const int which = n >= a.first[2] ? 2 : n >= a.first[1] ? 1 : 0;
    const PrepareArgs::One& o = a.one[which];
    const uint64_t local = n - a.first[which];
    const uint64_t row = local >> 32 ? local / o.groups : static_cast<uint32_t>(local) / o.groups;
    const uint32_t col = static_cast<uint32_t>(local - row * o.groups) * 8;
    const T* from = static_cast<const T*>(o.from) + row * o.ld_from + col;
    uint16_t* to = o.to + row * o.ld_to + col;
    if constexpr (sizeof(T) == 2) {
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < o.cols ? from[i] : 0;
        *reinterpret_cast<uint4*>(to) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
    } else {
        float v[8];
        if (o.vectors && col + 8 <= o.cols) {
            *reinterpret_cast<float4*>(v) = reinterpret_cast<const float4*>(from)[0];
            *reinterpret_cast<float4*>(v + 4) = reinterpret_cast<const float4*>(from)[1];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = col + i < o.cols ? from[i] : 0.0f;
        }
        uint32_t planes[3][4];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            uint32_t lo[3], hi[3];
            split3(v[i], lo);
            split3(v[i + 1], hi);
#pragma unroll
            for (int j = 0; j < 3; ++j) planes[j][i / 2] = lo[j] | hi[j] << 16;
        }
#pragma unroll
        for (int j = 0; j < 3; ++j)
            *reinterpret_cast<uint4*>(to + j * o.plane) = make_uint4(planes[j][0], planes[j][1], planes[j][2], planes[j][3]);
    }
}

// Adds the splits' sums in their order and rounds once.
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const Product q, T* out, T* out2, uint64_t ld, uint32_t rows, uint32_t cols) {
    const uint32_t groups = (cols + 3) / 4;
    const uint64_t n = blockIdx.x * 256ull + threadIdx.x;
    const uint64_t row = n / groups;
    const uint32_t col = static_cast<uint32_t>(n % groups) * 4;
    if (row >= q.rows_partial) return;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t s = 0; s < q.splits; ++s) {
        const float4 v = *reinterpret_cast<const float4*>(q.partial + (s * q.rows_partial + row) * q.ld_partial + col);
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    T* to = (row < rows ? out + row * ld : out2 + (row - rows) * ld) + col;
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < cols) to[i] = from_float<T>(v[i]);
}

// ---- host side -----------------------------------------------------------------------------------------------------

uint64_t round256(uint64_t n) { return (n + 255) & ~255ull; }
uint32_t planes_of(int dtype) { return dtype == CDMA_F32 ? 3 : 1; }
bool needs_copy(uint64_t ld, uint64_t rows, int dtype) { return dtype == CDMA_F32 || (rows > 1 && ld % 8 != 0); }

// Where things lie in the workspace behind the result words, and how the products are cut.
struct Plan {
    uint64_t grads, x, wg, wu, dx_partial, dw_partial, end;
    Product dx, dw;
};
constexpr uint32_t kProductCols = 256;
constexpr uint32_t kLeastSteps = 8;      // of an item: fewer would be lost in filling and emptying the pipeline

Plan plan_of(uint64_t m, uint64_t k, uint64_t f, uint64_t ld_x, uint64_t ld_wg, uint64_t ld_wu, int dtype, bool backward, bool dx, bool dw) {
    Plan l{};
    const uint64_t copy = 2 * planes_of(dtype), products = dtype == CDMA_F32 ? 6 : 1;
    l.grads = kFfnWsHeader;
    l.x = l.grads + (backward ? round256(2 * m * pitch_of(f) * copy) : 0);
    l.wg = l.x + (needs_copy(ld_x, m, dtype) ? round256(m * pitch_of(k) * copy) : 0);
    l.wu = l.wg + (needs_copy(ld_wg, f, dtype) ? round256(f * pitch_of(k) * copy) : 0);
    l.dx_partial = l.wu + (needs_copy(ld_wu, f, dtype) ? round256(f * pitch_of(k) * copy) : 0);
    l.dw_partial = l.end = l.dx_partial;
    if (!backward) return l;
    l.dx = Product{dx ? tiles_of(m, kTileRows) : 0, tiles_of(k, kProductCols), tiles_of(f, kStep), static_cast<uint32_t>(2 * products), 1, nullptr, pitch_of(k), m};
    l.dw = Product{dw ? 2 * tiles_of(f, kTileRows) : 0, tiles_of(k, kProductCols), tiles_of(m, kStep), static_cast<uint32_t>(products), 1, nullptr, pitch_of(k), 2 * f};
    // an even share of all steps for each pair of SMs: longer tiles are cut to about that
    uint64_t all = 0;
    for (const Product* q : {&l.dx, &l.dw}) all += static_cast<uint64_t>(q->tile_rows) * q->tile_cols * q->steps * q->parts;
    const uint64_t share = all / kPairs > kLeastSteps ? all / kPairs : kLeastSteps;
    for (Product* q : {&l.dx, &l.dw}) {
        const uint64_t steps = static_cast<uint64_t>(q->steps) * q->parts;
        if (steps >= 2 * share) q->splits = static_cast<uint32_t>(steps / share < 32 ? steps / share : 32);
    }
    l.dw_partial = l.dx_partial + (l.dx.splits > 1 && dx ? round256(l.dx.splits * l.dx.rows_partial * l.dx.ld_partial * 4) : 0);
    l.end = l.dw_partial + (l.dw.splits > 1 && dw ? round256(l.dw.splits * l.dw.rows_partial * l.dw.ld_partial * 4) : 0);
    return l;
}

template <bool GATE, uint32_t COLS, typename T, int ACT, typename Args>
cudaError_t launch_kernel(const CUtensorMap (&maps)[4], const Args& a, uint64_t items, const LaunchCtl& ctl, cudaStream_t stream) {
    auto kernel = ffn_mma_kernel<GATE, COLS, T, ACT, Args>;
    const cudaError_t e = opt_in_shared_memory(reinterpret_cast<const void*>(kernel), kSharedBytes<T, COLS>);
    if (e != cudaSuccess) return e;
    const uint32_t pairs = items < kPairs ? static_cast<uint32_t>(items) : kPairs;
    kernel<<<2 * pairs, kThreads, kSharedBytes<T, COLS>, stream>>>(maps[0], maps[1], maps[2], maps[3], a, ctl);
    count_kernel_launch();
    return cudaGetLastError();
}

// Hidden columns of a gate tile: the choice whose rounds over the pairs cost least.  A step of a narrow tile costs
// more for each column (it brings as many rows of x), so it pays only where wide tiles leave pairs idle.
uint32_t gate_cols(uint32_t tile_rows, uint32_t f) {
    uint32_t best = 256;
    double least = 0;
    for (const auto& [cols, cost] : {std::pair<uint32_t, double>{256, 1.0}, {128, 0.58}, {64, 0.36}}) {
        const uint64_t items = static_cast<uint64_t>(tile_rows) * tiles_of(f, cols / 2);
        const double t = cost * static_cast<double>((items + kPairs - 1) / kPairs);
        if (least == 0 || t < least) { least = t; best = cols; }
    }
    return best;
}

template <typename T, uint32_t COLS>
cudaError_t launch_gate(CUtensorMap (&maps)[4], GateArgs a, const Matrix& wg, const Matrix& wu, const LaunchCtl& ctl, cudaStream_t stream) {
    a.tile_cols = tiles_of(a.p.f, COLS / 2);
    if (!make_operand_map(&maps[2], wg, a.p.dtype, COLS / 2) || !make_operand_map(&maps[3], wu, a.p.dtype, COLS / 2)) return cudaErrorInvalidValue;
    const uint64_t items = static_cast<uint64_t>(a.tile_rows) * a.tile_cols;
    if (a.p.activation == CDMA_ACT_RELU) return launch_kernel<true, COLS, T, CDMA_ACT_RELU>(maps, a, items, ctl, stream);
    if (a.p.activation == CDMA_ACT_SILU) return launch_kernel<true, COLS, T, CDMA_ACT_SILU>(maps, a, items, ctl, stream);
    return launch_kernel<true, COLS, T, CDMA_ACT_GELU>(maps, a, items, ctl, stream);
}

template <typename T>
cudaError_t join(const Product& q, void* out, void* out2, uint64_t ld, uint32_t rows, uint32_t cols, cudaStream_t stream) {
    const uint64_t n = q.rows_partial * ((cols + 3) / 4);
    join_kernel<T><<<static_cast<uint32_t>((n + 255) / 256), 256, 0, stream>>>(q, static_cast<T*>(out), static_cast<T*>(out2), ld, rows, cols);
    count_kernel_launch();
    return cudaGetLastError();
}

// Copies the operands that need it; x, wg and wu then name what the kernels read.
template <typename T>
void prepare_operands(const FfnProblem& p, const uint64_t (&at)[3], Matrix (&m)[3], cudaStream_t stream) {
    uint8_t* ws = reinterpret_cast<uint8_t*>(p.ws);
    m[0] = {p.x, p.m, p.k, p.ld_x, 1};
    m[1] = {p.wg, p.f, p.k, p.ld_wg, 1};
    m[2] = {p.wu, p.f, p.k, p.ld_wu, 1};
    PrepareArgs prepare{};
    int count = 0;
    for (int i = 0; i < 3; ++i) {
        Matrix& o = m[i];
        if (!needs_copy(o.ld, o.rows, p.dtype)) continue;
        const uint64_t pitch = pitch_of(o.cols);
        const uint32_t groups = tiles_of(o.cols, 8);
        prepare.one[count] = {o.p, reinterpret_cast<uint16_t*>(ws + at[i]), o.ld, pitch, o.rows * pitch, static_cast<uint32_t>(o.rows),
                              static_cast<uint32_t>(o.cols), groups, o.ld % 4 == 0};
        prepare.first[count + 1] = prepare.first[count] + o.rows * groups;
        ++count;
        o = Matrix{ws + at[i], o.rows, o.cols, pitch, planes_of(p.dtype)};
    }
    if (count == 0) return;
    for (int i = count + 1; i < 4; ++i) prepare.first[i] = prepare.first[count];
    using Raw = typename std::conditional<sizeof(T) == 4, float, uint16_t>::type;
    prepare_kernel<Raw><<<static_cast<uint32_t>((prepare.first[3] + 255) / 256), 256, 0, stream>>>(prepare);
    count_kernel_launch();
}

template <typename T>
cudaError_t launch_all(const FfnProblem& p, bool backward, const LaunchCtl& ctl, cudaStream_t stream) {
    Plan l = plan_of(p.m, p.k, p.f, p.ld_x, p.ld_wg, p.ld_wu, p.dtype, backward, p.dx != nullptr, p.dwg != nullptr);
    uint8_t* ws = reinterpret_cast<uint8_t*>(p.ws);
    Matrix operands[3];
    prepare_operands<T>(p, {l.x, l.wg, l.wu}, operands, stream);
    const Matrix &x = operands[0], &wg = operands[1], &wu = operands[2];
    if (!backward && p.dtype != CDMA_F32 && p.m <= kFewRows) {
        FfnProblem few = p;
        few.x = x.p, few.wg = wg.p, few.wu = wu.p;
        few.ld_x = x.ld, few.ld_wg = wg.ld, few.ld_wu = wu.ld;
        return launch_ffn_stream(few, ctl, stream);
    }

    CUtensorMap maps[4];
    const uint64_t pitch = pitch_of(p.f);
    const Matrix grads{ws + l.grads, p.m, p.f, pitch, 2 * planes_of(p.dtype)};
    GateArgs g{p, tiles_of(p.m, kTileRows), 0, tiles_of(p.k, kStep), backward, {reinterpret_cast<uint16_t*>(ws + l.grads), pitch}};
    if (!make_operand_map(&maps[0], x, p.dtype, 128)) return cudaErrorInvalidValue;
    maps[1] = maps[0];
    const uint32_t cols = gate_cols(g.tile_rows, p.f);
    cudaError_t e = cols == 256   ? launch_gate<T, 256>(maps, g, wg, wu, ctl, stream)
                    : cols == 128 ? launch_gate<T, 128>(maps, g, wg, wu, ctl, stream)
                                  : launch_gate<T, 64>(maps, g, wg, wu, ctl, stream);
    if (e != cudaSuccess || !backward) return e;

    ProductsArgs a{p, l.dx, l.dw};
    a.dx.partial = reinterpret_cast<float*>(ws + l.dx_partial);
    a.dw.partial = reinterpret_cast<float*>(ws + l.dw_partial);
    if (!make_operand_map(&maps[0], x, p.dtype, kStep) || !make_operand_map(&maps[1], grads, p.dtype, kStep) || !make_operand_map(&maps[2], wg, p.dtype, kStep) ||
        !make_operand_map(&maps[3], wu, p.dtype, kStep))
        return cudaErrorInvalidValue;
    const uint64_t items = static_cast<uint64_t>(a.dx.tile_rows) * a.dx.tile_cols * a.dx.splits +
                           static_cast<uint64_t>(a.dw.tile_rows) * a.dw.tile_cols * a.dw.splits;
    e = launch_kernel<false, kProductCols, T, 0>(maps, a, items, ctl, stream);
    if (e == cudaSuccess && p.dx != nullptr && a.dx.splits > 1) e = join<T>(a.dx, p.dx, nullptr, p.ld_dx, p.m, p.k, stream);
    if (e == cudaSuccess && p.dwg != nullptr && a.dw.splits > 1) e = join<T>(a.dw, p.dwg, p.dwu, p.ld_dw, p.f, p.k, stream);
    return e;
}

}  // namespace

// Enough for every choice of gradients: leaving one out can cut the other finer.
uint64_t ffn_mma_workspace(uint64_t m, uint64_t k, uint64_t f, uint64_t ld_x, uint64_t ld_wg, uint64_t ld_wu, int dtype, bool backward) {
    const uint64_t both = plan_of(m, k, f, ld_x, ld_wg, ld_wu, dtype, backward, true, true).end;
    const uint64_t one = plan_of(m, k, f, ld_x, ld_wg, ld_wu, dtype, backward, true, false).end;
    const uint64_t other = plan_of(m, k, f, ld_x, ld_wg, ld_wu, dtype, backward, false, true).end;
    const uint64_t most = one > other ? one : other;
    return both > most ? both : most;
}

cudaError_t launch_ffn_mma(const FfnProblem& p, bool backward, const LaunchCtl& ctl, cudaStream_t stream) {
    timing_before_launch(stream);
    const cudaError_t e = p.dtype == CDMA_F32   ? launch_all<float>(p, backward, ctl, stream)
                          : p.dtype == CDMA_F16 ? launch_all<__half>(p, backward, ctl, stream)
                                                : launch_all<__nv_bfloat16>(p, backward, ctl, stream);
    timing_after_launch(stream);
    return e;
}

}  // namespace cdma
