// The dropout mask as a function: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", SC 2011) of the counter (col / 8, row, sequence low, sequence high) under the key (seed low,
// seed high).  Its four words are the eight 16-bit lanes of the elements 8*(col/8) .. +7 of the row, low half of a
// word first; an element whose lane is below `threshold` is dropped.  One generator call serves eight elements: a
// word for each element would make 2-byte tensors bound by the generator's multiplies instead of memory, and 16
// bits resolve the drop rate to 1/65536.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace cdma {

struct DropoutSpec {
    uint32_t threshold;   // elements with a lane below it are dropped: 0 none ... 65536 all
    float scale;          // 65536 / (65536 - threshold), 0 when everything is dropped
    uint32_t seq_lo, seq_hi;
    uint32_t keys[20];    // the ten rounds' pairs: operands of the rounds as they lie among the kernel's arguments
};

// False when p is not a number in [0, 1].
inline bool make_dropout_spec(double p, uint64_t seed, uint64_t sequence, DropoutSpec* out) {
    if (!(p >= 0.0 && p <= 1.0)) return false;
    out->threshold = static_cast<uint32_t>(p * 65536.0 + 0.5);
    out->scale = out->threshold < 65536u ? 65536.0f / static_cast<float>(65536u - out->threshold) : 0.0f;
    for (uint32_t round = 0; round < 10; ++round) {
        out->keys[2 * round] = static_cast<uint32_t>(seed) + round * 0x9E3779B9u;
        out->keys[2 * round + 1] = static_cast<uint32_t>(seed >> 32) + round * 0xBB67AE85u;
    }
    out->seq_lo = static_cast<uint32_t>(sequence);
    out->seq_hi = static_cast<uint32_t>(sequence >> 32);
    return true;
}

// The generator's block for elements 8*block .. +7 of the row.
struct DropoutLanes {
    uint32_t words[4];
    // element j of the eight is kept
    __device__ __forceinline__ bool kept(const DropoutSpec& d, int j) const {
        return (j & 1 ? words[j >> 1] >> 16 : words[j >> 1] & 0xffffu) >= d.threshold;
    }
};
__device__ __forceinline__ DropoutLanes dropout_lanes(const DropoutSpec& d, uint32_t row, uint32_t block) {
    uint32_t c0 = block, c1 = row, c2 = d.seq_lo, c3 = d.seq_hi;
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p0 = static_cast<uint64_t>(c0) * 0xD2511F53u, p1 = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        c0 = static_cast<uint32_t>(p1 >> 32) ^ c1 ^ d.keys[2 * round];
        c1 = static_cast<uint32_t>(p1);
        c2 = static_cast<uint32_t>(p0 >> 32) ^ c3 ^ d.keys[2 * round + 1];
        c3 = static_cast<uint32_t>(p0);
    }
    return DropoutLanes{{c0, c1, c2, c3}};
}

// Bit j set: element 8*block + j of the row is kept.
__device__ __forceinline__ uint32_t dropout_keep8(const DropoutSpec& d, uint32_t row, uint32_t block) {
    const DropoutLanes lanes = dropout_lanes(d, row, block);
    uint32_t keep = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) keep |= (lanes.kept(d, j) ? 1u : 0u) << j;
    return keep;
}

}  // namespace cdma
