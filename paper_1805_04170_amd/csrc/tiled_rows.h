// Rows of tiled tensors as the token operators' kernels walk them: the pieces that two grids of one tensor have in common along
// a row, and 16-byte vectors inside them.
#pragma once
#include "block_table.h"
#include "tensor_tiling_tokens.h"
#include "tt_wave.h"

namespace tt {

// A row is segments of `seg` columns, each inside one block of either grid (cuts halve, so the narrower block's width divides
// the other's), a segment `vps` vectors.
struct Pieces {
    uint32_t seg;  // columns per segment
    uint32_t vps;  // vectors per segment
    uint32_t tail; // values of a segment's last vector, 0: a whole one
    uint32_t nvec; // vectors per row
};

inline Pieces pieces_of(const BlockTable &a, const BlockTable &b, int64_t cols, int ev)
{
    Pieces s;
    s.seg = a.scols < b.scols ? a.scols : b.scols;
    s.vps = (s.seg + ev - 1) / ev;
    s.tail = s.seg % ev;
    s.nvec = (uint32_t)(cols / s.seg) * s.vps;
    return s;
}

// the first n values of a vector
template <typename T> __device__ __forceinline__ u32x4 load_part(const T *p, uint32_t n)
{
    uint32_t w[4] = {0, 0, 0, 0};
    for (uint32_t i = 0; i < n; ++i) {
        if constexpr (sizeof(T) == 2) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
        else w[i] = __float_as_uint(p[i]);
    }
    return u32x4{w[0], w[1], w[2], w[3]};
}
template <typename T> __device__ __forceinline__ void store_part(T *p, u32x4 v, uint32_t n)
{
    for (uint32_t i = 0; i < n; ++i) {
        if constexpr (sizeof(T) == 2) p[i] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
        else p[i] = __uint_as_float(v[i]);
    }
}

// the place in the table of the block that holds (row, col), and how many values into a shard that is
__device__ __forceinline__ size_t block_of(const BlockTable &b, uint32_t row, uint32_t col, size_t *offset)
{
    const uint32_t rb = row / b.srows, cb = col / b.scols;
    *offset = (size_t)(row - rb * b.srows) * b.scols + (col - cb * b.scols);
    return (size_t)(rb * b.nC + cb) * b.nrep;
}

// column and length of vector j of a row
__device__ __forceinline__ void vector_of(const Pieces &s, int ev, uint32_t j, uint32_t *col, uint32_t *n)
{
    const uint32_t q = j / s.vps, i = j - q * s.vps;
    *col = q * s.seg + i * ev;
    *n = i + 1 == s.vps && s.tail ? s.tail : (uint32_t)ev;
}

// into every replica
template <typename T>
__device__ __forceinline__ void store_all(const BlockTable &b, uint32_t row, uint32_t col, uint32_t n, u32x4 v)
{
    size_t at;
    const size_t blk = block_of(b, row, col, &at);
    for (uint32_t x = 0; x < b.nrep; ++x) {
        T *p = static_cast<T *>(b.p[blk + x]) + at;
        if (n == (uint32_t)kVec<T>) store16(p, v);
        else store_part(p, v, n);
    }
}

template <typename T> __device__ __forceinline__ const T *source_of(const BlockTable &b, uint32_t row, uint32_t col)
{
    size_t at;
    const size_t blk = block_of(b, row, col, &at);
    return static_cast<const T *>(b.p[blk]) + at;
}
template <typename T> __device__ __forceinline__ u32x4 load_vector(const T *p, uint32_t n) { return n == (uint32_t)kVec<T> ? load16(p) : load_part(p, n); }

template <typename I> __device__ __forceinline__ int64_t token_at(const void *ids, size_t i) { return (int64_t) static_cast<const I *>(ids)[i]; }

} // namespace tt
