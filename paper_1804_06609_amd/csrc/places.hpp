// Which bytes a strided tensor takes up, and whether two of them have any in common.  Host only; nothing here throws.
#pragma once
#include <stdint.h>

namespace dba {

typedef __int128 wide_t;

// Pieces of `len` bytes at `at` + sum of index * stride, three axes at most.
struct Places {
    uintptr_t at = 0;
    int64_t len = 0;
    int axes = 0;
    int64_t count[3], stride[3];       // counts above 1, by stride, greatest first
    wide_t extent = 0;                 // from the first byte to the last

    Places() {}
    Places(const void *at_, int64_t len_) : at(reinterpret_cast<uintptr_t>(at_)), len(len_), extent(len_) {}

    Places &axis(int64_t n, int64_t s)
    {
        if (n <= 1) return *this;
        int i = axes++;
        for (; i > 0 && stride[i - 1] < s; --i) {
            count[i] = count[i - 1];
            stride[i] = stride[i - 1];
        }
        count[i] = n;
        stride[i] = s;
        extent += (wide_t)s * (n - 1);
        return *this;
    }

    // Nested: every stride is at least what the axes below it span.  (So no two pieces overlap.)
    bool nested() const
    {
        wide_t below = len;
        for (int i = axes - 1; i >= 0; --i) {
            if (stride[i] < below) return false;
            below += (wide_t)stride[i] * (count[i] - 1);
        }
        return true;
    }

    bool fits() const { return extent <= (wide_t)1 << 62; }        // no stride is negative where this is asked
};

inline wide_t div_floor(wide_t a, wide_t b) { return a / b - (a % b < 0); }

// Axes i on of a from address pa, j on of b from pb, which span ea and eb.  Of equal outermost strides only the difference of the indexes counts, and
// few differences bring the rest within reach; else the greater stride's indexes that do are gone through.
inline bool places_meet(const Places &a, int i, wide_t pa, wide_t ea, const Places &b, int j, wide_t pb, wide_t eb, int &steps)
{
    while (i < a.axes && !a.stride[i]) ++i;
    while (j < b.axes && !b.stride[j]) ++j;
    if (pa + ea <= pb || pb + eb <= pa) return false;
    if (i == a.axes && j == b.axes) return true;
    const bool same = i < a.axes && j < b.axes && a.stride[i] == b.stride[j];
    if (!same && (i == a.axes || (j < b.axes && b.stride[j] > a.stride[i]))) return places_meet(b, j, pb, eb, a, i, pa, ea, steps);
    const wide_t s = a.stride[i], ra = ea - s * (a.count[i] - 1), rb = same ? eb - s * (b.count[j] - 1) : eb;
    // pa + x s + ra > pb and pa + x s < pb + rb
    const wide_t least = same ? -(wide_t)(b.count[j] - 1) : 0, most = a.count[i] - 1;
    const wide_t x0 = div_floor(pb - pa - ra, s) + 1, x1 = div_floor(pb + rb - 1 - pa, s);
    for (wide_t x = x0 > least ? x0 : least; x <= (x1 < most ? x1 : most); ++x) {
        if (--steps < 0 || places_meet(a, i + 1, pa + x * s, ra, b, j + same, pb, rb, steps)) return true;
    }
    return false;
}

// Whether any byte is in both.  Exact, but for tensors that interleave in strides of their own more often than `steps` times, which count as meeting.
inline bool meet(const Places &a, const Places &b, int steps = 1 << 16)
{
    const wide_t pa = (wide_t)a.at, pb = (wide_t)b.at;
    if (!a.len || !b.len || pa + a.extent <= pb || pb + b.extent <= pa) return false;
    return places_meet(a, 0, pa, a.extent, b, 0, pb, b.extent, steps);
}

}  // namespace dba
