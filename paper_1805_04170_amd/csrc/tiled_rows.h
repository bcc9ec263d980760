// Rows of tiled tensors as the token operators' kernels walk them: the pieces that two grids of one tensor have in common along
// a row, and 16-byte vectors inside them.
#pragma once
#include "block_table.h"
#include "tensor_tiling_tokens.h"
#include "tt_wave.h"

namespace tt {

// A row is `nseg` segments of `seg` columns, each inside one block of either grid (cuts halve, so the narrower block's width
// divides the other's), a segment `vps` vectors.
struct Pieces {
    uint32_t seg, nseg;
    uint32_t vps;              // vectors per segment
    uint32_t tail;             // values of a segment's last vector, 0: a whole one
    uint32_t a_shift, b_shift; // log2 of the segments in a block of the one grid and of the other
};

inline Pieces pieces_of(const BlockTable &a, const BlockTable &b, int64_t cols, int ev)
{
    Pieces s;
    s.seg = a.scols < b.scols ? a.scols : b.scols;
    s.nseg = (uint32_t)(cols / s.seg);
    s.vps = (s.seg + ev - 1) / ev;
    s.tail = s.seg % ev;
    s.a_shift = (uint32_t)__builtin_ctz(a.scols / s.seg);
    s.b_shift = (uint32_t)__builtin_ctz(b.scols / s.seg);
    return s;
}

__device__ __forceinline__ uint32_t quotient(uint32_t n, const Divisor &v) { return v.d == 1 ? n : __umulhi(n, v.m) >> (v.s - 1); }

// where segment q of a row begins in a grid whose blocks hold 2^shift segments a row: the block's first replica in the table, and
// the values in front of it in the shard
struct Place { uint32_t block; size_t at; };
__device__ __forceinline__ Place place_of(const BlockTable &b, const Pieces &s, uint32_t shift, uint32_t row, uint32_t q)
{
    const uint32_t rb = b.nR == 1 ? 0 : quotient(row, b.by_srows), cb = q >> shift;
    return {(rb * b.nC + cb) * b.nrep, (size_t)(row - rb * b.srows) * b.scols + (size_t)(q - (cb << shift)) * s.seg};
}
template <typename T> __device__ __forceinline__ const T *source_of(const BlockTable &b, const Pieces &s, uint32_t shift, uint32_t row, uint32_t q)
{
    const Place p = place_of(b, s, shift, row, q);
    return static_cast<const T *>(b.p[p.block]) + p.at;
}
// values of vector j of a segment (0 past its end)
__device__ __forceinline__ uint32_t values_of(const Pieces &s, uint32_t ev, uint32_t j) { return j >= s.vps ? 0 : j + 1 == s.vps && s.tail ? s.tail : ev; }

// the first n values of a vector
template <typename T> __device__ __forceinline__ u32x4 load_part(const T *p, uint32_t n)
{
    uint32_t w[4] = {0, 0, 0, 0};
    for (uint32_t i = 0; i < n; ++i) {
        if constexpr (sizeof(T) == 2) w[i >> 1] |= (uint32_t)load1(p + i) << (16 * (i & 1));
        else w[i] = __float_as_uint(load1(p + i));
    }
    return u32x4{w[0], w[1], w[2], w[3]};
}
template <typename T> __device__ __forceinline__ void store_part(T *p, u32x4 v, uint32_t n)
{
    for (uint32_t i = 0; i < n; ++i) {
        if constexpr (sizeof(T) == 2) store1(p + i, (uint16_t)(v[i >> 1] >> (16 * (i & 1))));
        else store1(p + i, __uint_as_float(v[i]));
    }
}

template <typename T> __device__ __forceinline__ void store_vector(T *p, u32x4 v, uint32_t n)
{
    if (n == (uint32_t)kVec<T>) store16(p, v);
    else store_part(p, v, n);
}
// the n values that begin `at` into a segment, into every replica
template <typename T> __device__ __forceinline__ void store_all(const BlockTable &b, const Place &to, uint32_t at, uint32_t n, u32x4 v)
{
    for (uint32_t x = 0; x < b.nrep; ++x) store_vector(static_cast<T *>(b.p[to.block + x]) + to.at + at, v, n);
}


template <typename I> __device__ __forceinline__ int64_t token_at(const void *ids, size_t i) { return (int64_t)load1(static_cast<const I *>(ids) + i); }
// ... at an index that all lanes share
template <typename I> __device__ __forceinline__ int64_t token_scalar(const void *ids, size_t i) { return (int64_t)load_scalar(static_cast<const I *>(ids) + i); }

} // namespace tt
