// Whether two matrices in memory share a byte.  Plain C++: the tests compile it for the host.
#pragma once

#include <cstdint>

namespace dcnn {

// Rows of `width` bytes, `ld` bytes apart (ld >= width; of a single row any).
struct Bytes {
    const char* name;
    const void* p;
    int64_t rows, ld, width;
};

// sum of floor((a * i + b) / m) over i < n, none of them negative: as many lattice points below a line, counted by Euclid's steps.
inline __int128 floor_sum(__int128 n, __int128 m, __int128 a, __int128 b) {
    __int128 sum = 0;
    for (;;) {
        if (a >= m) sum += n * (n - 1) / 2 * (a / m), a %= m;
        if (b >= m) sum += n * (b / m), b %= m;
        const __int128 top = a * n + b;
        if (top < m) return sum;
        n = top / m, b = top % m;
        const __int128 t = m;
        m = a, a = t;
    }
}

// Exact, also for matrices that lie in one another's gaps (columns of one wide buffer).  Row i of A meets row j of B where
// j * ldB lies in the open interval (d + i * ldA - widthB, d + i * ldA + widthA), d = A - B; the integers j of all these intervals are
// counted.  They move up with i, so those that meet rows 0 .. rowsB - 1 belong to i in one range.
inline bool overlap(const Bytes& a, const Bytes& b) {
    if (a.p == nullptr || b.p == nullptr || a.rows < 1 || b.rows < 1 || a.width < 1 || b.width < 1) return false;
    typedef __int128 I;
    const I d = (I)reinterpret_cast<uintptr_t>(a.p) - (I)reinterpret_cast<uintptr_t>(b.p);
    const I wa = a.width, wb = b.width, la = a.rows > 1 ? (I)a.ld : wa, lb = b.rows > 1 ? (I)b.ld : wb;
    const I end_a = d + (a.rows - 1) * la + wa, end_b = (b.rows - 1) * lb + wb;
    if (end_a <= 0 || d >= end_b) return false;
    // (la, lb > 0) the first i whose interval reaches 0 and the last one that begins below rowsB * ldB
    I first = 0, last = a.rows - 1;
    if (1 - wa - d > 0) first = (1 - wa - d + la - 1) / la;
    if ((end_b - d + la - 1) / la - 1 < last) last = (end_b - d + la - 1) / la - 1;
    if (first > last) return false;
    I from = d + first * la - wb, shift = 0;                   // both sums moved up by whole ldB, so that nothing is negative
    if (from < 0) shift = (-from + lb - 1) / lb * lb;
    return floor_sum(last - first + 1, lb, la, from + shift + wb + wa - 1) > floor_sum(last - first + 1, lb, la, from + shift);
}

}  // namespace dcnn
