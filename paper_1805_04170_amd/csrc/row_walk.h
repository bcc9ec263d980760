// Rows of one or two grids as 16-byte vectors, for kernels that hold a row (or a part of it) in registers: where a lane's vectors lie,
// loads that do not depend on a lane, stores into every replica.
#pragma once
#include "tiled_rows.h"

namespace tt {

// The vectors of a row, counted over the segments that the two grids have in common.
struct RowShape {
    Pieces s;
    uint32_t units; // vectors of a row
    Divisor by_vps;
    uint32_t cols;
};
inline RowShape row_shape(const BlockTable &a, const BlockTable &b, int64_t cols, int ev)
{
    RowShape r;
    r.s = pieces_of(a, b, cols, ev);
    r.units = r.s.nseg * r.s.vps;
    r.by_vps = divisor(r.s.vps);
    r.cols = (uint32_t)cols;
    return r;
}
// segments of less than a vector are taken value by value
inline bool narrow_segments(const RowShape &r, int ev) { return r.s.seg < (uint32_t)ev; }

// Vector j of a row: segment q, `at` values into it, n values, the first `dup` of which are another lane's as well.  A segment's short
// last vector is a whole one that ends with the segment, and a lane past the row's end has a vector that is another one's
// altogether (dup = EV): both compute and write the same, so that no access depends on a lane.
struct Spot { uint32_t q, at, n, dup; };
template <uint32_t EV> __device__ __forceinline__ Spot spot_of(const RowShape &r, uint32_t j)
{
    if (j >= r.units) return {0, 0, r.s.seg < EV ? r.s.seg : EV, EV};
    const uint32_t q = r.s.nseg == 1 ? 0 : quotient(j, r.by_vps), i = j - q * r.s.vps;
    if (i + 1 < r.s.vps || r.s.tail == 0) return {q, i * EV, EV, 0};
    if (r.s.seg < EV) return {q, 0, r.s.seg, 0};
    return {q, r.s.seg - EV, EV, EV - r.s.tail};
}

// Where a spot lies in a grid, in front of a row's begin (CUT: the row's block as well)
struct Lane { uint32_t block; size_t at; };
template <bool CUT> __device__ __forceinline__ Lane lane_of(const BlockTable &b, const Pieces &s, uint32_t shift, uint32_t row, const Spot &v)
{
    if constexpr (CUT) {
        const Place p = place_of(b, s, shift, row, v.q);
        return {p.block, p.at + v.at};
    } else {
        return {0, (size_t)row * b.scols + v.at};
    }
}

// NARROW: segments of less than a vector
template <typename T, bool NARROW> __device__ __forceinline__ u32x4 load_spot(const BlockTable &b, const Lane &l, const Spot &v)
{
    const T *p = static_cast<const T *>(b.p[l.block]) + l.at;
    if constexpr (NARROW) return load_part(p, v.n);
    else return load16(p);
}
template <typename T, bool CUT, bool NARROW> __device__ __forceinline__ void store_spot(const BlockTable &b, const Lane &l, const Spot &v, u32x4 w, bool once = false)
{
    auto one = [&](uint32_t x) {
        T *p = static_cast<T *>(b.p[l.block + x]) + l.at;
        if constexpr (NARROW) store_part(p, w, v.n);
        else if (once) store16_once(p, w);
        else store16(p, w);
    };
    one(0); // (outside of the loop: the compiler's waits count the stores that are sure to be made)
    if constexpr (CUT) {
        for (uint32_t x = 1; x < b.nrep; ++x) one(x);
    }
}

// which of the kernels' forms a launch takes
inline bool uncut(const BlockTable &b) { return b.nR * b.nC * b.nrep == 1; }

} // namespace tt
