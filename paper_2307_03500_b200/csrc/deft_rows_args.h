// Argument checks that the C-ABI entry points of the row operators share.  Host code.
#pragma once
#include <cmath>
#include <cstdint>
#include <utility>

#include "deft_rows.cuh"

namespace deft {

inline bool type_ok(int32_t t) { return t == DEFT_F32 || t == DEFT_BF16 || t == DEFT_F16; }
inline bool fits_f32(double x) { return std::isfinite((float)x); }   // what the kernels multiply by is fp32: no product with an infinity
inline bool elem_aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// A [rows, cols] matrix of a type: its pitch reaches over a row, its base is aligned to the element.
inline bool matrix_ok(const void* p, int32_t type, int64_t rows, int64_t cols, int64_t ld) {
    return p && ld >= cols && ld <= (1LL << 60) / rows && elem_aligned(p, type_bytes(type));   // offsets fit 64 bits
}

// Rows of a matrix in bytes.
struct Span { uintptr_t base; uint64_t row, pitch; };
inline Span span_of(const void* p, int32_t type, int64_t cols, int64_t ld, int64_t rows) {
    const uint64_t row = (uint64_t)cols * type_bytes(type);
    return Span{reinterpret_cast<uintptr_t>(p), row, rows == 1 ? row : (uint64_t)ld * type_bytes(type)};
}

// Whether two matrices of `rows` rows share a byte of their elements (columns of one buffer, or rows between each other's,
// do not).
inline bool overlap(Span a, Span b, int64_t rows) {
    if (a.base > b.base) std::swap(a, b);
    const uint64_t apart = b.base - a.base, last = (uint64_t)(rows - 1);
    if (apart >= last * a.pitch + a.row) return false;
    if (a.pitch == b.pitch) {            // every row of b lies `at` behind a's row `below` further down
        const uint64_t below = apart / a.pitch, at = apart % a.pitch;
        return at < a.row || (at + b.row > a.pitch && below < last);
    }
    // both lists of rows ascend: the later of two rows that do not meet waits for the other list's next one
    for (uint64_t i = 0, j = 0; i <= last && j <= last;) {
        const uint64_t x = i * a.pitch, y = apart + j * b.pitch;
        if (x + a.row <= y) ++i;
        else if (y + b.row <= x) ++j;
        else return true;
    }
    return false;
}

// Whether y may be written while `in` is read: apart, or element for element the same place.
inline bool in_place_or_apart(Span y, Span in, bool same_type, int64_t rows) {
    return (y.base == in.base && y.pitch == in.pitch && same_type) || !overlap(y, in, rows);
}

}  // namespace deft
