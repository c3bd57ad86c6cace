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
    uint32_t seed_lo, seed_hi, seq_lo, seq_hi;
};

// False when p is not a number in [0, 1].
inline bool make_dropout_spec(double p, uint64_t seed, uint64_t sequence, DropoutSpec* out) {
    if (!(p >= 0.0 && p <= 1.0)) return false;
    out->threshold = static_cast<uint32_t>(p * 65536.0 + 0.5);
    out->scale = out->threshold < 65536u ? 65536.0f / static_cast<float>(65536u - out->threshold) : 0.0f;
    out->seed_lo = static_cast<uint32_t>(seed);
    out->seed_hi = static_cast<uint32_t>(seed >> 32);
    out->seq_lo = static_cast<uint32_t>(sequence);
    out->seq_hi = static_cast<uint32_t>(sequence >> 32);
    return true;
}

// Bit j set: element 8*block + j of the row is kept.
__device__ __forceinline__ uint32_t dropout_keep8(const DropoutSpec& d, uint32_t row, uint32_t block) {
    uint32_t c0 = block, c1 = row, c2 = d.seq_lo, c3 = d.seq_hi, k0 = d.seed_lo, k1 = d.seed_hi;
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p0 = static_cast<uint64_t>(c0) * 0xD2511F53u, p1 = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        c0 = static_cast<uint32_t>(p1 >> 32) ^ c1 ^ k0;
        c1 = static_cast<uint32_t>(p1);
        c2 = static_cast<uint32_t>(p0 >> 32) ^ c3 ^ k1;
        c3 = static_cast<uint32_t>(p0);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
    uint32_t keep = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        keep |= ((w[j] & 0xffffu) >= d.threshold ? 1u : 0u) << (2 * j);
        keep |= ((w[j] >> 16) >= d.threshold ? 1u : 0u) << (2 * j + 1);
    }
    return keep;
}

}  // namespace cdma
