// Whether tables of rows, and tensors of three strides, overlap (host only).
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


// Runs of `bytes` bytes in three dimensions, each with its number of places and the bytes from one to the next (any: none, or backwards).  What lies nowhere (NULL) or
// has no places shares nothing.
struct Strided {
    const void* at;
    int64_t n[3], apart[3], bytes;
    __int128 from, to;                                                // the first byte, and the one behind the last
    Strided(const void* at, int64_t n0, int64_t apart0, int64_t n1, int64_t apart1, int64_t n2, int64_t apart2, int64_t bytes)
        : at(at), n{n0, n1, n2}, apart{apart0, apart1, apart2}, bytes(bytes), from((uintptr_t)at), to(from) {
        if (!at || bytes < 1 || n0 < 1 || n1 < 1 || n2 < 1) return;
        to += bytes;
        for (int i = 0; i < 3; ++i) (apart[i] < 0 ? from : to) += (__int128)(n[i] - 1) * apart[i];
    }
    Strided(const void* at, int64_t bytes) : Strided(at, 1, 0, 1, 0, 1, 0, bytes) {}
};
// The same as runs that do not touch, the widest steps first.
struct Runs {
    typedef __int128 wide;
    int rank = 0;
    wide n[3], apart[3], bytes, reach[4];                             // reach: bytes from the first to behind the last, of dimensions i and on
    explicit Runs(const Strided& s) : bytes(s.bytes) {
        for (int i = 0; i < 3; ++i) {
            const wide step = s.apart[i] < 0 ? -(wide)s.apart[i] : (wide)s.apart[i];
            if (s.n[i] == 1 || step == 0) continue;
            int at = rank++;
            for (; at > 0 && apart[at - 1] < step; --at) { apart[at] = apart[at - 1]; n[at] = n[at - 1]; }
            apart[at] = step;
            n[at] = s.n[i];
        }
        while (rank > 0 && apart[rank - 1] <= bytes) { --rank; bytes += (n[rank] - 1) * apart[rank]; }
        for (int i = rank - 2; i >= 0; --i)
            if (apart[i] == apart[i + 1] * n[i + 1]) {
                n[i] *= n[i + 1];
                apart[i] = apart[i + 1];
                --rank;
                for (int k = i + 1; k < rank; ++k) { n[k] = n[k + 1]; apart[k] = apart[k + 1]; }
            }
        reach[rank] = bytes;
        for (int i = rank - 1; i >= 0; --i) reach[i] = reach[i + 1] + (n[i] - 1) * apart[i];
    }
};
// the least and the greatest k with -before < d + k step < behind, of 0 <= lo .. hi
inline bool steps_between(__int128 d, __int128 step, __int128 before, __int128 behind, __int128& lo, __int128& hi) {
    const auto down = [](__int128 n, __int128 by) { return n / by - (n % by < 0); };
    const __int128 first = down(-before - d, step) + 1, last = down(behind - 1 - d, step);
    if (first > lo) lo = first;
    if (last < hi) hi = last;
    return lo <= hi;
}
// Dimensions i and on of a, and j and on of b, `d` bytes behind.  Blocks that are equally far apart meet by the difference of their numbers; else those of the one whose
// steps are wider are taken one by one, as far as they reach into the other.
inline bool runs_share(const Runs& a, int i, const Runs& b, int j, __int128 d) {
    if (d >= a.reach[i] || -d >= b.reach[j]) return false;
    if (i == a.rank && j == b.rank) return true;
    if (i < a.rank && j < b.rank && a.apart[i] == b.apart[j]) {
        __int128 lo = 1 - a.n[i], hi = b.n[j] - 1;
        if (steps_between(d, a.apart[i], b.reach[j + 1], a.reach[i + 1], lo, hi))
            for (__int128 k = lo; k <= hi; ++k) if (runs_share(a, i + 1, b, j + 1, d + k * a.apart[i])) return true;
        return false;
    }
    if (j < b.rank && (i == a.rank || a.apart[i] < b.apart[j])) {
        __int128 lo = 0, hi = b.n[j] - 1;
        if (steps_between(d, b.apart[j], b.reach[j + 1], a.reach[i], lo, hi))
            for (__int128 k = lo; k <= hi; ++k) if (runs_share(a, i, b, j + 1, d + k * b.apart[j])) return true;
        return false;
    }
    return runs_share(b, j, a, i, -d);
}
// Whether they share a byte.
inline bool share(const Strided& a, const Strided& b) {
    if (a.from >= a.to || b.from >= b.to || a.to <= b.from || b.to <= a.from) return false;
    return runs_share(Runs(a), 0, Runs(b), 0, b.from - a.from);
}

}  // namespace accerl
