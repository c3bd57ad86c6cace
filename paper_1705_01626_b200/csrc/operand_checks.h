// Argument checks of operators whose operands are matrices with a row stride.
#pragma once

#include <cstdint>

namespace cdma {

struct Operand {
    uintptr_t at;
    uint64_t rows, cols, ld, size;   // ld in elements, size in bytes per element
    uint64_t span() const { return rows == 0 || cols == 0 ? 0 : ((rows - 1) * ld + cols) * size; }
};

// ld = 0 stands for dense rows.  False: a null pointer where there are elements, a stride shorter than a row, or a
// span past 2^48 bytes.
inline bool make_operand(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t size, Operand* out) {
    if (ld == 0) ld = cols;
    if (ld < cols || ld > (1ull << 40)) return false;
    if (rows != 0 && cols != 0 && (p == nullptr || ld > (1ull << 48) / size / rows)) return false;
    *out = Operand{reinterpret_cast<uintptr_t>(p), rows, cols, ld, size};
    return true;
}

inline bool starts_on_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline bool same_place(const Operand& a, const Operand& b) {
    return a.at == b.at && a.size == b.size && (a.ld == b.ld || a.rows <= 1);
}

// Whether two operands may share a byte.  Column ranges of one wider buffer (equal strides, disjoint columns) do not.
inline bool overlap(const Operand& a, const Operand& b) {
    if (a.span() == 0 || b.span() == 0 || a.at + a.span() <= b.at || b.at + b.span() <= a.at) return false;
    if (a.ld * a.size != b.ld * b.size) return true;
    const uint64_t pitch = a.ld * a.size;
    const uint64_t shift = b.at >= a.at ? (b.at - a.at) % pitch : (pitch - (a.at - b.at) % pitch) % pitch;
    return !(shift >= a.cols * a.size && shift + b.cols * b.size <= pitch);
}

}  // namespace cdma
