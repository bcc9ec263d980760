// The shards of a tensor as the token operators' kernels take them: one pointer per block of the tile grid (flattening
// theorem, Sec. 4.4 of arXiv 1805.04170), replicas one after the other, and the pieces that two grids of one tensor have in
// common along a row.
#pragma once
#include <cstdint>
#include "tt_internal.h"

namespace tt {

// n / d for n below 2^31 by one multiplication: with 2^(s-1) < d <= 2^s and m = ceil(2^(31+s) / d) the excess m d - 2^(31+s) is below
// d <= 2^s, and n times it below 2^(31+s).
struct Divisor { uint32_t d, m, s; };
inline Divisor divisor(uint32_t d)
{
    Divisor v{d, 0, 0};
    while ((uint64_t(1) << v.s) < d) ++v.s;
    if (d > 1) v.m = (uint32_t)(((uint64_t(1) << (31 + v.s)) + d - 1) / d);
    return v;
}

struct BlockTable {
    void *p[kMaxShards]; // block (r, c), replica x at (r * nC + c) * nrep + x
    uint32_t nR, nC, nrep;
    uint32_t srows, scols; // shard extent
    Divisor by_srows;
};

// false: an uneven cut.  Entries are NULL where the list is (a size query needs the geometry alone).
inline bool make_blocks(const void *const *shards, const tt_tiling &t, int k, int64_t rows, int64_t cols, BlockTable *b)
{
    Grid g;
    if (!make_grid(t.cut, k, rows, cols, &g)) return false;
    b->nR = 1u << g.kR;
    b->nC = 1u << g.kC;
    b->nrep = 1u << g.kX;
    b->srows = (uint32_t)g.srows;
    b->scols = (uint32_t)g.scols;
    b->by_srows = divisor(b->srows ? b->srows : 1);
    for (uint32_t i = 0; i < (uint32_t)kMaxShards; ++i) b->p[i] = nullptr;
    for (uint32_t s = 0; s < (1u << k); ++s) {
        const uint32_t r = extract(s, g.maskR, k), c = extract(s, g.maskC, k), x = extract(s, g.maskX, k);
        b->p[(r * b->nC + c) * b->nrep + x] = shards ? const_cast<void *>(shards[s]) : nullptr;
    }
    return true;
}

// every shard is there and aligned to its elements (a tensor without values has no buffers)
inline bool shards_fit(const void *const *shards, int k, int elem_bytes, bool empty = false)
{
    if (!shards || empty) return shards != nullptr;
    for (int s = 0; s < (1 << k); ++s)
        if (!shards[s] || reinterpret_cast<uintptr_t>(shards[s]) % (uintptr_t)elem_bytes) return false;
    return true;
}
inline bool aligned_to(const void *p, int bytes) { return p && reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

// extents that the kernels count in 32 bits
inline bool fits31(int64_t v) { return v < (int64_t(1) << 31); }

inline bool valid_dtype(int d) { return d == TT_F32 || d == TT_BF16; }
inline int dtype_bytes(int d) { return d == TT_BF16 ? 2 : 4; }

} // namespace tt
