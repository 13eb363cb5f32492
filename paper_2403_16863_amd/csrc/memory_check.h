// Whether two tensors with strides share an element: for the checks of outputs at the C entries.
#pragma once
#include <stdint.h>

// rows * columns elements of 2 bytes, row r at data + r * stride elements.
struct Rows2D {
    const void* data;
    long long rows, columns, stride;
};

// Bytes from the first element to behind the last (the sizes are within limits that keep this in 64 bits).
inline unsigned long long span_bytes(const Rows2D& t) { return 2ull * ((t.rows > 1 ? (unsigned long long)(t.rows - 1) * t.stride : 0) + t.columns); }

inline bool bytes_meet(const void* a, unsigned long long an, const void* b, unsigned long long bn) {
    return a && b && (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}

// Whether columns [0, an) at a and [0, bn) at b, in rows of one stride, meet in some row.
inline bool columns_meet(const void* a, long long an, const void* b, long long bn, long long stride) {
    const long long bytes = 2 * stride, gap = (long long)((uintptr_t)b - (uintptr_t)a) % bytes;
    const long long at = gap < 0 ? gap + bytes : gap;  // where b's columns begin in a's rows
    return at < 2 * an || at + 2 * bn > bytes;
}

// Matrices of one stride (a single row has any) may lie beside each other in the rows of a wider one; others whose ranges meet are taken to overlap.
inline bool rows_meet(const Rows2D& a, const Rows2D& b) {
    if (!a.data || !b.data || !bytes_meet(a.data, span_bytes(a), b.data, span_bytes(b))) return false;
    if ((a.rows > 1 && b.rows > 1 && a.stride != b.stride) || (a.rows == 1 && b.rows == 1)) return true;
    return columns_meet(a.data, a.columns, b.data, b.columns, a.rows > 1 ? a.stride : b.stride);
}
