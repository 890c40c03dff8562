// Whether two matrices in memory share a byte, from their addresses, rows and
// strides alone.  Host code only, free of HIP headers.
#pragma once

#include <cstdint>

namespace rtcc {
namespace kern {

// `rows` rows of `width` bytes, `stride` bytes apart.
struct Extent {
    int64_t at, rows, stride, width;
    int64_t end() const { return at + (rows - 1) * stride + width; }
};
inline Extent extent(const void *p, int64_t rows, int64_t stride, int64_t width, int64_t elem) {
    Extent e{int64_t(reinterpret_cast<uintptr_t>(p)), p ? rows : 0, stride * elem, width * elem};
    // rows that follow each other are one
    if (e.rows == 1 || (e.rows > 1 && e.stride == e.width)) e.width *= e.rows, e.rows = 1, e.stride = e.width;
    return e;
}

// Whether a row of b shares a byte with [at, at + width).
inline bool row_overlaps(int64_t at, int64_t width, const Extent &b) {
    if (b.rows == 0) return false;
    const int64_t d = at - b.at;
    // the first row that ends behind `at`
    const int64_t j = d < b.width ? 0 : (d - b.width) / b.stride + 1;
    return j < b.rows && j * b.stride < d + width;
}

// Exact where either's rows follow each other or both have one stride.  Others, that
// lie between each other's rows, are known to overlap by their first and last rows.
inline bool overlap(const Extent &a, const Extent &b) {
    if (a.rows == 0 || b.rows == 0 || a.at >= b.end() || b.at >= a.end()) return false;
    if (a.rows == 1) return row_overlaps(a.at, a.width, b);
    if (b.rows == 1) return row_overlaps(b.at, b.width, a);
    if (a.stride == b.stride)  // row i of a is as far from row j of b as row 0 from row j - i
        return row_overlaps(a.at, a.width, {b.at - (a.rows - 1) * b.stride, a.rows + b.rows - 1, b.stride, b.width});
    auto ends = [](const Extent &x, const Extent &y) {
        return row_overlaps(x.at, x.width, y) || row_overlaps(x.at + (x.rows - 1) * x.stride, x.width, y);
    };
    return ends(a, b) || ends(b, a);
}

}  // namespace kern
}  // namespace rtcc
