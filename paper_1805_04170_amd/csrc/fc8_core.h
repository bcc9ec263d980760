// Products of 8-bit integers, X W^T with K contiguous in both: operands as they are tiled, and a tile on v_mfma_i32_16x16x64_i8.
//
// A K tile is 128 bytes of a row, as a K tile of 64 is in bf16: fragments, LDS layout, swizzle and the order of a k-step are those
// of gemm_mma.h, and a k-step multiplies twice as many values in the time.  Sums are whole numbers and exact, so neither K's
// cuts nor the order of the K tiles change a result.
#pragma once
#include <cstdint>
#include "block_table.h"
#include "gemm_core.h"
#include "gemm_core2.h"
#include "gemm_mma.h"
#include "tt_wave.h"

namespace tt {
namespace fc8 {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int BK8 = 128; // values of a K tile

// One operand: its rows are cut into blocks of `srows`, K into blocks of whole segments.
struct Operand {
    const void *p[kMaxShards];
    uint32_t row_blocks, srows;      // blocks along the rows
    Divisor by_srows;
    uint32_t row_stride, k_stride;   // places in p from a block to the next one along the rows, along K
    uint32_t k_shift;                // log2 of the segments in a block
    uint32_t pitch;                  // bytes from row to row
    uint32_t rows;
};

// The K of the product: `segments` pieces of `seg` values, each inside one block of either operand, `tiles` K tiles a piece.  A piece
// ends inside its last K tile where seg is no multiple of 128: the operand whose blocks are the pieces has zeros there, and what the
// other one has does not matter.
struct Steps8 {
    uint32_t segments, seg, tiles;
    Divisor by_tiles;
    uint32_t all; // segments * tiles
};

// a K tile: segment and the tile in it
struct At { uint32_t seg, tile; };
__device__ __forceinline__ At at_tile(const Steps8 &s, uint32_t t)
{
    if (s.segments == 1) return {0, t};
    const uint32_t q = s.by_tiles.d == 1 ? t : __umulhi(t, s.by_tiles.m) >> (s.by_tiles.s - 1);
    return {q, t - q * s.tiles};
}

// first value of row r in segment q; `most`: the last offset from there at which 16 bytes of the row's memory lie
struct RowAt { const char *p; uint32_t most; };
__device__ __forceinline__ RowAt row_at(const Operand &o, const Steps8 &s, uint32_t r, uint32_t q)
{
    const uint32_t rb = o.row_blocks == 1 ? 0 : (o.by_srows.d == 1 ? r : __umulhi(r, o.by_srows.m) >> (o.by_srows.s - 1));
    const uint32_t kb = q >> o.k_shift, in = (q - (kb << o.k_shift)) * s.seg;
    return {static_cast<const char *>(o.p[rb * o.row_stride + kb * o.k_stride]) + (size_t)(r - rb * o.srows) * o.pitch + in, o.pitch - 16 - in};
}

// The K tiles of ROWS rows of an operand on their way into LDS, by NT threads: chunk c = tid + NT i of a tile is row c / 8, position
// c % 8, and holds the row's chunk position ^ ((row >> 1) & 7).  Rows from `end` on are the last row again: they feed results that are
// never stored.
//   kInside     the rows lie in one block and no K tile passes a row's end, so the address is a scalar and an offset
//   kToTheEnd   ... but K tiles may pass the row's end: lanes behind it fetch the tile's first bytes instead
//   kAnywhere   rows of any block
enum { kAnywhere = 0, kToTheEnd = 1, kInside = 2 };
template <int ROWS, int NT, int ONE> struct Feed {
    static constexpr int NL = ROWS * 8 / NT;
    static_assert(NL >= 1 && (NT / 8) % 16 == 0, "the swizzle is the same for all of a thread's chunks");
    uint32_t voff[ONE ? NL : 1];
    uint64_t base;
    const char *row[ONE ? 1 : NL];
    uint32_t most, row0, end, kc, tile;
    At at;
    __device__ __forceinline__ void bind(const Operand &o, const Steps8 &s)
    {
        if constexpr (ONE) {
            const RowAt x = row_at(o, s, row0, at.seg);
            base = core2::uniform64(x.p) + (uint64_t)at.tile * BK8;
            most = uniform(x.most);
        } else {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const uint32_t r = row0 + (threadIdx.x >> 3) + NT / 8 * i;
                const RowAt x = row_at(o, s, r < end ? r : end - 1, at.seg);
                row[i] = x.p;
                most = x.most;
            }
        }
    }
    __device__ __forceinline__ void begin(const Operand &o, const Steps8 &s, uint32_t first_row, uint32_t end_row, uint32_t first)
    {
        row0 = first_row;
        end = end_row;
        tile = first;
        at = at_tile(s, tile);
        kc = ((threadIdx.x & 7) ^ ((threadIdx.x >> 4) & 7)) * 16;
        if constexpr (ONE) {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const uint32_t r = row0 + (threadIdx.x >> 3) + NT / 8 * i;
                voff[i] = ((r < end ? r : end - 1) - row0) * o.pitch + kc;
            }
        }
        bind(o, s);
    }
    // `by` K tiles further
    __device__ __forceinline__ void next(const Operand &o, const Steps8 &s, uint32_t by)
    {
        tile += by;
        at.tile += by;
        if (at.tile < s.tiles) {
            if constexpr (ONE) base += by * BK8;
        } else {
            at = at_tile(s, tile);
            bind(o, s);
        }
    }
    __device__ __forceinline__ void issue(int i, uint32_t lds) const
    {
        const uint32_t to = lds + core2::wave2() * 1024u + (uint32_t)i * (NT * 16u);
        if constexpr (ONE == kInside) {
            dev::lds_dma16(voff[i], base, to);
        } else if constexpr (ONE == kToTheEnd) {
            dev::lds_dma16(at.tile * BK8 + kc <= most ? voff[i] : voff[i] - kc, base, to);
        } else {
            const uint32_t off = at.tile * BK8 + kc;
            dev::lds_dma16(row[i] + (off < most ? off : most), to);
        }
    }
};

template <int TM, int TN> struct Frags8 { i32x4 a[TM], b[TN]; };
template <int ROWS, int T> struct Reader8 {
    mma::Reader<ROWS, true, T> r;
    __device__ __forceinline__ void init(int w0, int lane) { r.init(w0, lane); }
    __device__ __forceinline__ i32x4 read(const char *tile, int ks, int i) const { return __builtin_bit_cast(i32x4, r.read(tile, ks, i)); }
};

// acc += cur.a cur.b, and meanwhile nxt = the fragments of k-step ks of the tiles At, Bt, and NLOAD calls issue(0 ..): reads in the
// first half of the slots of two MFMAs, loads into LDS in the second (gemm_mma.h)
template <int NLOAD, class RA, class RB, int TM, int TN, class Issue>
__device__ __forceinline__ void k_step8(i32x4 (&acc)[TM][TN], const Frags8<TM, TN> &cur, Frags8<TM, TN> &nxt, const RA &ra, const RB &rb,
                                        const char *At, const char *Bt, int ks, Issue &&issue)
{
    constexpr int MM = TM * TN, SL = MM / 2, RD = TM + TN, RS = SL / 2, L0 = SL / 2, LS = SL - L0;
    static_assert(MM % 2 == 0 && SL >= 2, "slots");
    int mm = 0, rd = 0, ld = 0;
#pragma unroll
    for (int s = 0; s < SL; ++s) {
        const int rto = s >= RS ? RD : (s + 1) * RD / RS, lto = s < L0 ? 0 : (s - L0 + 1) * NLOAD / LS;
#pragma unroll
        for (; rd < rto; ++rd) {
            if (rd < TN) nxt.b[rd] = rb.read(Bt, ks, rd);
            else nxt.a[rd - TN] = ra.read(At, ks, rd - TN);
        }
#pragma unroll
        for (; ld < lto; ++ld) issue(ld);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (; mm < 2 * (s + 1); ++mm) { // rows of blocks back and forth: one operand of each MFMA is the one before's
            const int i = mm / TN, j = i & 1 ? TN - 1 - mm % TN : mm % TN;
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cur.b[j], cur.a[i], acc[i][j], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Sums over `count` K tiles (more than 0), first, first + by, .., of rows m0 .. m1 - 1 and channels n0 .. n1 - 1 of the
// result (of the tile from m0, n0 on).  WM x WN waves, each
// 16 TM x 16 TN; NS LDS stages, so that NS - 1 K tiles are on their way or being multiplied.  A lane ends up with row lane % 16 and
// four consecutive channels 4 (lane / 16) .. of every block.
template <int WM, int WN, int TM, int TN, int NS, int ONE> struct Tile8 {
    static constexpr int NT = WM * WN * 64, BM = WM * TM * 16, BN = WN * TN * 16;
    static constexpr int kA = BM * BK8, kB = BN * BK8, kStage = kA + kB;
    static constexpr size_t kSmem = NS * (size_t)kStage;
    typedef Feed<BM, NT, ONE> FA;
    typedef Feed<BN, NT, ONE> FB;
    static constexpr int LPS = FA::NL + FB::NL;
    static_assert(NS >= 2 && (NS - 1) * LPS < 64, "loads that a wait can count");
    i32x4 acc[TM][TN];
    __device__ __forceinline__ void run(const Operand &A, const Operand &B, const Steps8 &s, uint32_t m0, uint32_t m1, uint32_t n0, uint32_t n1, uint32_t first, uint32_t by, uint32_t count, char *smem)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const uint32_t lds0 = dev::lds_addr(smem);
        FA fa;
        FB fb;
        fa.begin(A, s, m0, m1, first);
        fb.begin(B, s, n0, n1, first);
        uint32_t left = count - 1; // K tiles behind the one that is fetched next; past the end the last one is fetched again
        auto issue = [&](int i, uint32_t stage) {
            if (i < FA::NL) fa.issue(i, stage);
            else fb.issue(i - FA::NL, stage + kA);
        };
        auto advance = [&]() {
            if (left > 0) {
                fa.next(A, s, by);
                fb.next(B, s, by);
                --left;
            }
        };
#pragma unroll
        for (int st = 0; st < NS; ++st) {
#pragma unroll
            for (int i = 0; i < LPS; ++i) issue(i, lds0 + (uint32_t)st * kStage);
            advance();
        }
        Reader8<BM, TM> ra;
        Reader8<BN, TN> rb;
        ra.init(wave / WN * (TM * 16), lane);
        rb.init(wave % WN * (TN * 16), lane);
        Frags8<TM, TN> f0, f1;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
        __builtin_amdgcn_s_waitcnt(mma::waitcnt_vm((NS - 1) * LPS)); // this wave's chunks of the first tile have landed
        __syncthreads();                                  // everyone's have
#pragma unroll
        for (int j = 0; j < TN; ++j) f0.b[j] = rb.read(smem + kA, 0, j);
#pragma unroll
        for (int i = 0; i < TM; ++i) f0.a[i] = ra.read(smem, 0, i);
        uint32_t cur = 0;
        for (uint32_t t = 0; t < count; ++t) {
            const char *At = smem + cur * kStage;
            k_step8<0>(acc, f0, f1, ra, rb, At, At + kA, 1, [](int) {});
            // this wave has read the tile, and its chunks of the next one have landed; then everyone's
            __builtin_amdgcn_s_waitcnt(mma::waitcnt_vm_lds((NS - 2) * LPS));
            __syncthreads();
            const uint32_t lds_free = lds0 + cur * kStage;
            cur = cur + 1 == NS ? 0 : cur + 1;
            const char *nA = smem + cur * kStage;
            k_step8<LPS>(acc, f1, f0, ra, rb, nA, nA + kA, 0, [&](int i) { issue(i, lds_free); });
            advance();
        }
        // what was fetched past the end has landed, and every wave is done with the stages
        __builtin_amdgcn_s_waitcnt(mma::waitcnt_vm_lds(0));
        __syncthreads();
    }
};

} // namespace fc8
} // namespace tt
