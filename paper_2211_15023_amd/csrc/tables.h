// Whether tables of rows overlap (host only).
#pragma once
#include <stdint.h>

namespace accerl {

// rows of `bytes` bytes each, `apart` bytes from one to the next (at least `bytes`)
struct Table { const void* at; int64_t rows, apart, bytes; };
inline Table table(const void* at, int64_t rows, int64_t ld, int64_t cols, int64_t element) { return {at, rows, ld * element, cols * element}; }
inline Table table(const void* at, int64_t bytes) { return {at, at ? 1 : 0, bytes, bytes}; }
// Whether they share a byte.  Rows that lie between the other table's rows, as columns of one wider table do, share none.
inline bool share(const Table& a, const Table& b) {
    typedef __int128 wide;                                            // (strides may be anything)
    if (a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
    const wide at = (wide)(uintptr_t)a.at, bt = (wide)(uintptr_t)b.at, d = bt - at;
    if (d >= (wide)(a.rows - 1) * a.apart + a.bytes || -d >= (wide)(b.rows - 1) * b.apart + b.bytes) return false;
    const auto down = [](wide n, wide by) { return n / by - (n % by < 0); };
    if (a.apart == b.apart) {
        // row i of a and row i + k of b are d + k apart from each other: the least k that is not wholly before
        wide k = down(-b.bytes - d, a.apart) + 1;
        if (k < 1 - a.rows) k = 1 - a.rows;
        return k < b.rows && d + k * a.apart < a.bytes;
    }
    if (a.rows > b.rows) return share(b, a);
    for (int64_t i = 0; i < a.rows; ++i) {
        // the last row of b that begins before the end of a's row
        const wide from = at + (wide)i * a.apart;
        wide j = down(from + a.bytes - 1 - bt, b.apart);
        if (j >= b.rows) j = b.rows - 1;
        if (j >= 0 && bt + j * b.apart + b.bytes > from) return true;
    }
    return false;
}

}  // namespace accerl
