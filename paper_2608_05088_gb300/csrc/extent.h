// extent.h -- where a call's operands lie, and whether two of them share memory (host only).
#pragma once
#include <cstdint>

namespace malt {

// Where an operand lies: rows of `bytes`, `ld` bytes apart (a vector is a row).
struct Extent {
    const void* p = nullptr;
    int64_t rows = 0, bytes = 0, ld = 0;
};
inline Extent extent_of(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t size) {
    return {p, rows, cols * size, ld * size};
}
inline Extent extent_of(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }
// Whether they have a byte in common.  Columns of one wider matrix have none; operands between each other's
// rows at different strides are taken to.
inline bool overlap(const Extent& a, const Extent& b) {
    if (a.p == nullptr || b.p == nullptr || a.rows <= 0 || b.rows <= 0 || a.bytes <= 0 || b.bytes <= 0) return false;
    const int64_t at = reinterpret_cast<intptr_t>(a.p), bt = reinterpret_cast<intptr_t>(b.p);
    if (at + (a.rows - 1) * a.ld + a.bytes <= bt || bt + (b.rows - 1) * b.ld + b.bytes <= at) return false;
    if (a.rows == 1 && b.rows == 1) return true;
    if (a.rows > 1 && b.rows > 1 && a.ld != b.ld) return true;
    const int64_t ld = a.rows > 1 ? a.ld : b.ld, d = ((bt - at) % ld + ld) % ld;     // b's first column, of a's row
    return d < a.bytes || d + b.bytes > ld;
}

}  // namespace malt
