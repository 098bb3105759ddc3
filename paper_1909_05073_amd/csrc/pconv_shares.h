// How the workgroups of the register-tiled kernel share units of work, and whom they wait for.  Plain C++, so that a host
// program can play through every order in which the hardware may start them.
//
// A set of `takers` workgroups, j = 0 .. takers - 1, deals out the iterations (unit, chunk) of its units in equal contiguous
// ranges.  A piece is what a workgroup has of one unit.  One that ends before the unit does hands its sums on to workgroup
// j + 1; one that begins behind the unit's first chunk waits at its end for those of j - 1.  The piece that is handed on runs
// first, the one that is taken over last, so that j waits for j - 1 alone, and j - 1 at that point for lower ones of the same unit.
//
// Whoever waits keeps its place on the chip, so j - 1 must have its own by then.  The hardware starts the workgroups of a launch in order
// of their ids on each XCD (ids that are equal mod 8), and promises nothing from one XCD to the next: with two launches
// under way, one XCD may be full of the first and its neighbour of the second, and each of them waits for workgroups that cannot start
// before the other ends.  Sets within an XCD take j from the workgroup's id.  The set of all workgroups takes it from a counter
// that each asks when it starts (shares_by_ticket), so that lower ones have always started.
#pragma once

#include <cstdint>

#ifdef __HIP__
#define PCONV_ANYWHERE __host__ __device__ __forceinline__
#else
#define PCONV_ANYWHERE inline
#endif

namespace pconv {

// First and last unit that a workgroup touches, its first chunk of the one and the end of its chunks of the other.
struct UnitShare { int first, last, head_c0, tail_c1; };

struct UnitPiece { int unit, c_begin, c_end; };

// Whether workgroup j of `wgs` has a share, and which; units, n_chunks > 0.
PCONV_ANYWHERE bool unit_share(int j, int wgs, int units, int n_chunks, UnitShare &s)
{
    const int64_t iters = int64_t(units) * n_chunks;
    const int64_t takers = iters < wgs ? iters : wgs;                    // nobody gets an empty range in between
    if (j >= takers) return false;
    int64_t it0 = iters * j / takers, it1 = iters * (j + 1) / takers;
    // When every unit is shared by the same number P of workgroups, those finish their chunks at
    // the same time and then pass the sums on one after the other, each link of that chain taking
    // about as long as 2.5 chunks.  Their shares are therefore graded, the first the smallest and
    // 2.5 chunks more for each successor (boundary k at k n / P - 2.5 k (P - k) / 2), so that a
    // workgroup finishes about when its predecessor's sums arrive.
    const int P = int(takers / units);
    if (int64_t(units) * P == takers && P >= 2 && 4 * n_chunks >= P * (16 + 5 * (P - 1))) {
        const int u = j / P, kk = j - u * P;
        auto bound = [&](int q) { return (4 * q * n_chunks / P - 5 * q * (P - q)) / 4; };
        it0 = int64_t(u) * n_chunks + bound(kk);
        it1 = int64_t(u) * n_chunks + bound(kk + 1);
    }
    s.first = int(it0 / n_chunks);
    s.last = int((it1 - 1) / n_chunks);
    s.head_c0 = int(it0 - int64_t(s.first) * n_chunks);                  // > 0: the first unit begins elsewhere
    s.tail_c1 = int(it1 - int64_t(s.last) * n_chunks);                   // < n_chunks: the last unit ends elsewhere
    return true;
}

// A share's pieces, in the order in which they run: the one to hand on, whole units, the one taken over.
PCONV_ANYWHERE int unit_pieces(const UnitShare &s, int n_chunks)
{
    const bool head = s.head_c0 > 0, tail = s.tail_c1 < n_chunks;
    const int whole = s.last - s.first + 1 - (head ? 1 : 0) - (tail ? 1 : 0);
    return (tail ? 1 : 0) + (whole > 0 ? whole : 0) + (head && !(tail && s.first == s.last) ? 1 : 0);
}

PCONV_ANYWHERE UnitPiece unit_piece(const UnitShare &s, int n_chunks, int piece)
{
    const bool head = s.head_c0 > 0, tail = s.tail_c1 < n_chunks;
    const int first_whole = head ? s.first + 1 : s.first, whole = (tail ? s.last - 1 : s.last) - first_whole + 1, at = piece - (tail ? 1 : 0);
    if (tail && piece == 0) return UnitPiece{s.last, s.first == s.last ? s.head_c0 : 0, s.tail_c1};
    if (at < whole) return UnitPiece{first_whole + at, 0, n_chunks};
    return UnitPiece{s.first, s.head_c0, n_chunks};
}

// Whether j is a ticket (else the workgroup's id, within its XCD).
PCONV_ANYWHERE constexpr bool shares_by_ticket(bool one_set) { return one_set; }

}  // namespace pconv

#undef PCONV_ANYWHERE
