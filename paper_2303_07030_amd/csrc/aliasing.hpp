// Whether two arrays of a call share memory, rows with something between them included:
// the queries, keys and values of one projection lie between each other's rows.  Host only.
#pragma once

#include <algorithm>
#include <cstdint>
#include <utility>

namespace nsd {

// `rows` rows of `width` bytes, `ld` bytes from one to the next (no rows, no array: nothing).  An
// array that is written may be the one that is read with the same number in `same`, if that is
// not 0: the whole of it, at one address.
struct Area {
    const void *p;
    int64_t rows, width, ld;
    int same = 0;
};

inline Area flat_area(const void *p, int64_t bytes) { return Area{p, 1, bytes, bytes}; }

inline bool areas_meet(Area a, Area b) {
    using Wide = __int128;  // a distance times a number of rows may pass 64 bits
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
    auto end = [](const Area &x) { return (Wide)(x.rows - 1) * x.ld + x.width; };
    auto down = [](Wide x, Wide y) { return x >= 0 ? x / y : -((-x + y - 1) / y); };
    if (a.rows > b.rows) std::swap(a, b);
    // places are counted from a's first
    const Wide at = (Wide) reinterpret_cast<uintptr_t>(b.p) - (Wide) reinterpret_cast<uintptr_t>(a.p);
    if (at >= end(a) || at + end(b) <= 0) return false;
    if (a.rows > 1 && a.ld == b.ld) {  // row j of b: `rest` places behind row j + by of a
        const Wide by = down(at, a.ld), rest = at - by * a.ld;
        auto some = [&](Wide n) { return n < a.rows && n > -(Wide)b.rows; };
        return (rest < a.width && some(by)) || (rest + b.width > a.ld && some(by + 1));
    }
    for (int64_t i = 0; i < a.rows; ++i) {  // the rows of b that end behind this one's start
        const Wide lo = (Wide)i * a.ld, hi = lo + a.width;
        const Wide first = std::max<Wide>(down(lo - at - b.width, b.ld) + 1, 0);
        if (first < b.rows && at + first * b.ld < hi) return true;
    }
    return false;
}

}  // namespace nsd
