// Whether what a call writes overlaps what it reads.
#pragma once

#include <stdint.h>

namespace ps {

// Rows of so many elements of `size` bytes each, so far apart.
struct RowSet {
    const void* p;
    int64_t stride, width;
    int32_t size = 2;
};
// Whether nx rows of one set and ny of another share a byte.  Sets with one stride (parts of a buffer) are told apart by a
// division; others only if they lie interleaved, and then row by row.
inline bool rows_meet(const RowSet& x, int64_t nx, const RowSet& y, int64_t ny) {
    struct Span {
        int64_t at, step, bytes;
    };
    auto span = [](const RowSet& r, int64_t n) {       // by rising address
        Span s{(int64_t)reinterpret_cast<uintptr_t>(r.p), n > 1 ? r.size * r.stride : 0, r.size * r.width};
        if (s.step < 0) s.at += (n - 1) * s.step, s.step = -s.step;
        return s;
    };
    const Span a = span(x, nx), b = span(y, ny);
    if (a.at + (nx - 1) * a.step + a.bytes <= b.at || b.at + (ny - 1) * b.step + b.bytes <= a.at) return false;
    if (a.step == b.step && a.step > 0) {    // row i of a and row j of b meet if d - a.bytes < (i - j) step < d + b.bytes
        const int64_t d = b.at - a.at, low = d - a.bytes;
        int64_t k = low / a.step - (low % a.step < 0) + 1;
        if (k < 1 - ny) k = 1 - ny;
        return k < nx && k * a.step < d + b.bytes;
    }
    for (int64_t i = 0, j = 0; i < nx && j < ny;) {
        const int64_t s = a.at + i * a.step, t = b.at + j * b.step;
        if (s + a.bytes <= t) ++i;
        else if (t + b.bytes <= s) ++j;
        else return true;
    }
    return false;
}
inline bool rows_meet(const RowSet& x, const RowSet& y, int64_t n) { return rows_meet(x, n, y, n); }

}  // namespace ps
