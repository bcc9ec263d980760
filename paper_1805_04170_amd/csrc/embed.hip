// Embedding of tokens and its table's gradient, on tiled tensors: the rows of a table by token number in front of a chain of
// layers, and the sum of the rows' gradients by token number behind its backward pass.
//
// Both move rows and hardly compute: what bounds them is memory (the result is written once, every row read once) and, for a
// few tokens, the trip to a token's number and on to its row.  Forward, 16384 of 65536 x 4096 bf16 rows: 31.5 us, 5.9 TB/s; 16 rows 3.6 us
// on the GPU.  Gradient of a 65536 x 8192 table over 8 shards from 16384 tokens: 298 us, 4.5 TB/s, of it sorting 11, the rows 268 (0.27 GB
// read and 1.08 GB written: nothing twice), joining 17.
#include <algorithm>
#include <cstdint>
#include <type_traits>
#include "launch_util.h"
#include "block_table.h"
#include "tensor_tiling_tokens.h"
#include "tiled_rows.h"

namespace tt {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kU = 2;     // vectors per lane of a wave's part of a segment
constexpr int kRunBatch = 8, kRowBatch = 4, kPartials = 8; // rows, or partial sums, that are on their way together

// How the segments of a row are shared out.  Wide form: a part of kU vectors per lane to a wave, so that a wave's row, segment and
// addresses are scalars.  Narrow form: a vector per lane, a segment to 2^glog lanes (one, but for few tokens).  The wide form is the
// faster one even where it leaves most lanes idle (gradient of a 50000-row table from 8192 tokens, wide / narrow, us: width 8 25 / 35, 64 26 / 35, 192 27 / 42;
// forward alike), so the narrow one is for segments of less than a vector, and for few tokens, where a wave has nothing to look up and
// many narrow rows are one store (64 tokens, wide / narrow: width 8 15 / 11, 64 15 / 9, 192 16 / 11).
struct Split {
    Pieces s;
    uint32_t wide, glog;
    uint32_t parts; // of a segment (wide)
    Divisor by_row, by_segment, by_nseg; // parts of a row, of a segment; segments of a row
};

Split split_rows(const BlockTable &a, const BlockTable &b, int64_t cols, int ev, bool few)
{
    Split w;
    w.s = pieces_of(a, b, cols, ev);
    w.wide = few ? w.s.vps > 32 : w.s.seg >= (uint32_t)ev;
    w.glog = 0;
    while ((1u << w.glog) < w.s.vps && w.glog < 6) ++w.glog;
    w.parts = w.wide ? (w.s.vps + 64 * kU - 1) / (64 * kU) : 1;
    w.by_row = divisor(w.s.nseg * w.parts);
    w.by_segment = divisor(w.parts);
    w.by_nseg = divisor(w.s.nseg);
    return w;
}

// workgroups for `rows` rows
uint64_t groups_of(const Split &w, uint64_t rows)
{
    if (w.wide) return (rows * w.s.nseg * w.parts + kWaves - 1) / kWaves;
    return ((rows * w.s.nseg << w.glog) + kThreads - 1) / kThreads;
}

// a wave's work in the wide form, all of it scalars
struct WaveWork { uint32_t row, q, j0; };
__device__ __forceinline__ WaveWork wave_work(const Split &w, uint32_t group)
{
    const uint32_t g = group * kWaves + uniform(threadIdx.x >> 6);
    const uint32_t row = quotient(g, w.by_row), rest = g - row * w.by_row.d;
    const uint32_t q = quotient(rest, w.by_segment);
    return {row, q, (rest - q * w.parts) * 64 * kU};
}
// a lane's in the narrow form: vector j of a segment
struct LaneWork { uint32_t row, q, j; };
__device__ __forceinline__ LaneWork lane_work(const Split &w)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x, g = i >> w.glog, row = quotient(g, w.by_nseg);
    return {row, g - row * w.s.nseg, i & ((1u << w.glog) - 1)};
}
// ... where a segment is less than a vector: all of it
__device__ __forceinline__ LaneWork small_work(const Split &w)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x, row = quotient(i, w.by_nseg);
    return {row, i - row * w.s.nseg, 0};
}

// A wave's vectors of a segment, one per lane and u.  Every lane loads whole vectors, so that no load depends on a lane: a
// segment's last vector, where it is short, is the values that end with the segment (those in front of its own are its
// neighbour's too), lanes past the end take it as well; `own` says how many of a vector's last values are the lane's to store.
template <typename T> struct Columns {
    uint32_t col[kU], own[kU];
    __device__ __forceinline__ Columns(const Pieces &s, uint32_t j0)
    {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const uint32_t j = j0 + u * 64 + (threadIdx.x & 63u), last = s.seg - kVec<T>;
            own[u] = values_of(s, kVec<T>, j);
            col[u] = j * kVec<T> < last ? j * kVec<T> : last;
        }
    }
    // into every replica of a segment that begins at `to`; ONCE: store16_once
    template <bool ONCE> __device__ __forceinline__ void store(const BlockTable &b, const Place &to, int u, u32x4 v) const
    {
        if (own[u] == 0) return;
        for (uint32_t x = 0; x < b.nrep; ++x) {
            T *dst = static_cast<T *>(b.p[to.block + x]) + to.at + col[u];
            if (own[u] == (uint32_t)kVec<T>) {
                if constexpr (ONCE) store16_once(dst, v);
                else store16(dst, v);
                continue;
            }
#pragma unroll
            for (int i = 1; i < kVec<T>; ++i) {
                if ((uint32_t)i < kVec<T> - own[u]) continue;
                if constexpr (sizeof(T) == 2) store1(dst + i, (uint16_t)(v[i >> 1] >> (16 * (i & 1))));
                else store1(dst + i, __uint_as_float(v[i]));
            }
        }
    }
};

// Segments of less than a vector: value by value.
template <typename T> struct Small {
    uint32_t n;
    __device__ __forceinline__ explicit Small(const Pieces &s) : n(s.seg) {}
    __device__ __forceinline__ u32x4 load(const T *segment) const { return load_part(segment, n); }
    __device__ __forceinline__ void store(const BlockTable &b, const Place &to, u32x4 v) const
    {
        for (uint32_t x = 0; x < b.nrep; ++x) store_part(static_cast<T *>(b.p[to.block + x]) + to.at, v, n);
    }
    // fp32 values of the same columns
    __device__ __forceinline__ void load_floats(float (&f)[kVec<T>], const float *segment) const
    {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) f[i] = (uint32_t)i < n ? load1(segment + i) : 0.0f;
    }
    __device__ __forceinline__ void store_floats(const float (&f)[kVec<T>], float *segment) const
    {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i)
            if ((uint32_t)i < n) store1(segment + i, f[i]);
    }
};

// One vector of any segment (few tokens)
template <typename T> struct Column1 {
    uint32_t col, own;
    bool tiny;
    __device__ __forceinline__ Column1(const Pieces &s, uint32_t j) : own(values_of(s, kVec<T>, j)), tiny(s.seg < (uint32_t)kVec<T>)
    {
        const uint32_t last = tiny ? 0 : s.seg - kVec<T>;
        col = j * kVec<T> < last ? j * kVec<T> : last;
    }
    __device__ __forceinline__ u32x4 load(const T *segment) const { return tiny ? load_part(segment, own) : load16(segment + col); }
    __device__ __forceinline__ void store(const BlockTable &b, const Place &to, u32x4 v) const
    {
        if (own == 0) return;
        for (uint32_t x = 0; x < b.nrep; ++x) {
            T *dst = static_cast<T *>(b.p[to.block + x]) + to.at + col;
            if (own == (uint32_t)kVec<T>) store16(dst, v);
            else if (tiny) store_part(dst, v, own);
            else {
#pragma unroll
                for (int i = 1; i < kVec<T>; ++i) {
                    if ((uint32_t)i < kVec<T> - own) continue;
                    if constexpr (sizeof(T) == 2) store1(dst + i, (uint16_t)(v[i >> 1] >> (16 * (i & 1))));
                    else store1(dst + i, __uint_as_float(v[i]));
                }
            }
        }
    }
};

template <typename T> __device__ __forceinline__ u32x4 scaled(u32x4 v, float scale)
{
    float f[kVec<T>];
    unpack16(v, f, T());
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) f[i] *= scale;
    return pack16(f, T());
}

// ------------------------------------------------------------------------------------------------------- forward

struct EmbedParams {
    BlockTable W, X;
    Split w;
    const void *ids;
    uint32_t tokens;
    int64_t vocab;
    float scale;
};

// A wave's part of one token's row, all of it loaded before the first vector is stored.
template <typename T, typename I> __global__ __launch_bounds__(kThreads) void embed_wide_kernel(const EmbedParams p)
{
    const WaveWork g = wave_work(p.w, blockIdx.x);
    if (g.row >= p.tokens) return;
    const int64_t v = token_scalar<I>(p.ids, g.row);
    const Columns<T> c(p.w.s, g.j0);
    const Place to = place_of(p.X, p.w.s, p.w.s.b_shift, g.row, g.q);
    u32x4 r[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) r[u] = u32x4{0, 0, 0, 0};
    if (v >= 0 && v < p.vocab) {
        const T *src = source_of<T>(p.W, p.w.s, p.w.s.a_shift, (uint32_t)v, g.q);
#pragma unroll
        for (int u = 0; u < kU; ++u) r[u] = load16(src + c.col[u]);
#pragma unroll
        for (int u = 0; u < kU; ++u) r[u] = scaled<T>(r[u], p.scale);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) c.template store<true>(p.X, to, u, r[u]);
}

template <typename T, typename I> __global__ __launch_bounds__(kThreads) void embed_narrow_kernel(const EmbedParams p)
{
    const LaneWork g = small_work(p.w);
    const Small<T> c(p.w.s);
    if (g.row >= p.tokens) return;
    const int64_t v = token_at<I>(p.ids, g.row);
    u32x4 r = u32x4{0, 0, 0, 0};
    if (v >= 0 && v < p.vocab) r = scaled<T>(c.load(source_of<T>(p.W, p.w.s, p.w.s.a_shift, (uint32_t)v, g.q)), p.scale);
    c.store(p.X, place_of(p.X, p.w.s, p.w.s.b_shift, g.row, g.q), r);
}

// ------------------------------------------------------------------------------------------------------ backward
// Three launches.  (1) Tokens sorted by number, stably.  (2) Every row of the table's gradient: the sum over its tokens in order.
// Numbers with many tokens (more than `chunk`) would keep one wave busy long after the rest is done: the sorted list is cut into
// runs of `chunk`, and in the same launch each run adds up its part of such a number into a partial sum.  (3) The rows of
// those numbers: the sums over their partial sums.

// (1) Numbers are dealt out to workgroups like cards (frequent numbers are neighbours in most vocabularies): workgroup w sorts
// the tokens whose number is w modulo the workgroups' count, 2^wlog of them.  The list has w's numbers behind w - 1's, each
// workgroup's in increasing order: place(v) = (v mod 2^wlog) * range + v / 2^wlog numbers them so, and start[place(v)],
// start[place(v) + 1] enclose v's tokens.
//
// A workgroup reads all tokens, each wave a stretch of them.  It counts how many belong to workgroups before it (where its part
// of the list begins) and how often each of its numbers comes in each wave's stretch; after a scan over (number, wave) the
// waves walk their stretches again and put their tokens in place, in order.  No workgroup waits for another, whatever the
// numbers are.  Bound by trips to memory and LDS: 3000 tokens 6.5 us, 16384 11, 32768 20 (their numbers no longer fit the registers).
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortRange = 1024, kSortLoads = 16;

struct Places { uint32_t wlog, range; };
__device__ __forceinline__ uint32_t place(const Places &s, uint32_t v) { return (v & ((1u << s.wlog) - 1)) * s.range + (v >> s.wlog); }

struct SortParams {
    const void *ids;
    uint32_t tokens;
    Places to;
    int64_t vocab;
    uint32_t *order, *number, *start; // tokens and their numbers in the list's order; where a place's tokens begin
};

constexpr uint32_t kNoToken = ~0u;
// kSortLoads numbers a lane from tb on, kNoToken where there is none (all loads before the first number is looked at)
template <typename I> __device__ __forceinline__ void load_numbers(uint32_t (&v)[kSortLoads], const SortParams &p, uint32_t tb, uint32_t end)
{
    I raw[kSortLoads];
    const uint32_t t = tb + (threadIdx.x & 63u);
#pragma unroll
    for (int i = 0; i < kSortLoads; ++i) {
        const uint32_t at = t + i * 64 < end ? t + i * 64 : end - 1;
        raw[i] = load1(static_cast<const I *>(p.ids) + at);
    }
#pragma unroll
    for (int i = 0; i < kSortLoads; ++i) {
        const int64_t n = (int64_t)raw[i];
        v[i] = t + i * 64 < end && n >= 0 && n < p.vocab ? (uint32_t)n : kNoToken;
    }
}

template <typename I> __global__ __launch_bounds__(kSortThreads) void sort_tokens_kernel(const SortParams p)
{
    __shared__ uint32_t at[kSortWaves * kSortRange];
    __shared__ uint32_t part[2][kSortWaves];
    const uint32_t lane = threadIdx.x & 63u, w = uniform(threadIdx.x >> 6), me = blockIdx.x, range = p.to.range;
    const uint32_t groups = 1u << p.to.wlog;
    for (uint32_t i = threadIdx.x; i < kSortWaves * range; i += kSortThreads) at[i] = 0;
    __syncthreads();
    const uint32_t stretch = ((p.tokens + kSortThreads - 1) / kSortThreads) * 64;
    const uint32_t t0 = w * stretch < p.tokens ? w * stretch : p.tokens, t1 = t0 + stretch < p.tokens ? t0 + stretch : p.tokens;
    uint32_t *mine = at + w * range;
    uint32_t below = 0, v[kSortLoads];
    for (uint32_t tb = t0; tb < t1; tb += 64 * kSortLoads) {
        load_numbers<I>(v, p, tb, t1);
#pragma unroll
        for (int i = 0; i < kSortLoads; ++i) {
            if (v[i] == kNoToken) continue;
            const uint32_t who = v[i] & (groups - 1);
            below += who < me ? 1 : 0;
            if (who == me) wave::lds_add(&mine[v[i] >> p.to.wlog], 1);
        }
    }
    below = wave_sum(below);
    if (lane == 0) part[0][w] = below;
    __syncthreads();
    // thread r: the workgroup's r-th number; exclusive scan of the totals over the workgroup
    uint32_t total = 0, before = 0;
    if (threadIdx.x < range)
        for (uint32_t i = 0; i < (uint32_t)kSortWaves; ++i) total += at[i * range + threadIdx.x];
    uint32_t incl = total;
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
        const uint32_t o = wave::shfl_up(incl, by);
        if (lane >= (uint32_t)by) incl += o;
    }
    if (lane == 63) part[1][w] = incl;
    __syncthreads();
    for (uint32_t i = 0; i < (uint32_t)kSortWaves; ++i) before += part[0][i] + (i < w ? part[1][i] : 0);
    before += incl - total;
    if (threadIdx.x < range) {
        p.start[me * range + threadIdx.x] = before;
        uint32_t run = before;
        for (uint32_t i = 0; i < (uint32_t)kSortWaves; ++i) {
            const uint32_t c = at[i * range + threadIdx.x];
            at[i * range + threadIdx.x] = run;
            run += c;
        }
        if (me + 1 == groups && threadIdx.x + 1 == range) p.start[groups * range] = run;
    }
    __syncthreads();
    for (uint32_t tb = t0; tb < t1; tb += 64 * kSortLoads) {
        if (stretch > 64 * kSortLoads) load_numbers<I>(v, p, tb, t1); // (otherwise they are still here)
#pragma unroll
        for (int i = 0; i < kSortLoads; ++i) {
            const bool in = v[i] != kNoToken && (v[i] & (groups - 1)) == me;
            const uint32_t r = in ? v[i] >> p.to.wlog : 0;
            uint64_t left = wave::ballot(in);
            while (left) { // one number of the 64 tokens at a time
                const uint32_t n = wave::read_lane(r, __builtin_ctzll(left));
                const bool same = in && r == n;
                const uint64_t who = wave::ballot(same);
                const uint32_t to = mine[n];
                wave::fence();
                if (same) {
                    const uint32_t rank = (uint32_t)__builtin_popcountll(who & ((uint64_t(1) << lane) - 1));
                    p.order[to + rank] = tb + i * 64 + lane;
                    p.number[to + rank] = v[i];
                    if (rank == 0) mine[n] = to + (uint32_t)__builtin_popcountll(who);
                }
                wave::fence();
                left &= ~who;
            }
        }
    }
}

struct EmbedGradParams {
    BlockTable G, W; // the rows' gradients, the table's
    Split w;
    const void *ids;
    const uint32_t *order, *number, *start;
    float *partial; // [2 runs][cols]: run c's part of a number that began before the run, of one that begins inside it
    Places to;
    Divisor by_chunk;
    uint32_t places; // 2^wlog * range
    uint32_t tokens;
    uint32_t chunk, runs, cols;
    uint32_t run_groups; // workgroups for runs (wide)
    uint32_t rows, apart; // of the table's gradient per wave, and how far they lie from each other (wide)
    int64_t vocab;
    float scale;
};
__device__ __forceinline__ float *partial_of(const EmbedGradParams &p, uint32_t run, bool inside, uint32_t q)
{
    return p.partial + (size_t)(2 * run + (inside ? 1 : 0)) * p.cols + (size_t)q * p.w.s.seg;
}

// Where a wave's segment lies in the rows of the tokens' gradients.  Cuts by rows make the block a matter of the token;
// the lanes then hold the table of blocks (a scalar load per row would be a trip to memory per row).
template <typename T> struct Sources {
    const T *base; // nothing cut by rows: of token 0
    uint32_t lo, hi, block, at;
    __device__ __forceinline__ Sources(const EmbedGradParams &p, const WaveWork &g)
    {
        const uint32_t cb = g.q >> p.w.s.a_shift;
        at = (g.q - (cb << p.w.s.a_shift)) * p.w.s.seg;
        block = cb * p.G.nrep;
        base = static_cast<const T *>(p.G.p[block]) + at;
        lo = hi = 0;
        if (p.G.nR > 1) {
            const uint64_t mine = (uint64_t)(uintptr_t)p.G.p[threadIdx.x & 63u];
            lo = (uint32_t)mine;
            hi = (uint32_t)(mine >> 32);
        }
    }
    __device__ __forceinline__ const T *row(const EmbedGradParams &p, uint32_t t) const
    {
        if (p.G.nR == 1) return base + (size_t)t * p.G.scols;
        const uint32_t rb = quotient(t, p.G.by_srows), b = rb * p.G.nC * p.G.nrep + block;
        const uint64_t q = (uint64_t)wave::read_lane(hi, (int)b) << 32 | wave::read_lane(lo, (int)b);
        return reinterpret_cast<const T *>((uintptr_t)q) + (size_t)(t - rb * p.G.srows) * p.G.scols + at;
    }
};

// the sums of a wave's part of a segment
template <typename T> struct Sums {
    float f[kU][kVec<T>];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int u = 0; u < kU; ++u)
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) f[u][i] = 0.0f;
    }
    __device__ __forceinline__ void add(int u, u32x4 v)
    {
        float g[kVec<T>];
        unpack16(v, g, T());
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) f[u][i] += g[i];
    }
};

// n rows (all BATCH of them where n is larger) added to the sums in order, on their way together; token(k): the k-th
template <typename T, int BATCH, class F>
__device__ __forceinline__ void add_batch(Sums<T> &a, const EmbedGradParams &p, const Sources<T> &src, const Columns<T> &c, uint32_t n, F &&token)
{
    u32x4 r[BATCH][kU];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
        if ((uint32_t)k >= n) break;
        const T *from = src.row(p, token(k));
#pragma unroll
        for (int u = 0; u < kU; ++u) r[k][u] = load16(from + c.col[u]);
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
        if ((uint32_t)k >= n) break;
#pragma unroll
        for (int u = 0; u < kU; ++u) a.add(u, r[k][u]);
    }
}
// the rows of places [b, e) of the sorted list
template <typename T, int BATCH>
__device__ __forceinline__ void add_rows(Sums<T> &a, const EmbedGradParams &p, const Sources<T> &src, const Columns<T> &c, uint32_t b, uint32_t e)
{
    for (uint32_t w = b; w < e; w += 64) {
        const uint32_t mine = w + (threadIdx.x & 63u), tokens = mine < e ? p.order[mine] : 0, n = e - w < 64 ? e - w : 64;
        for (uint32_t i = 0; i < n; i += BATCH) add_batch<T, BATCH>(a, p, src, c, n - i, [&](int k) { return wave::read_lane(tokens, (int)i + k); });
    }
}

// What a run has to do with numbers of many tokens: it may end one at its first place and begin one at its last.
struct Run { uint32_t b, e, first, last; bool any; };
__device__ __forceinline__ Run run_of(const EmbedGradParams &p, uint32_t run)
{
    const uint32_t total = load_scalar(p.start + p.places), b = run * p.chunk;
    if (b >= total) return {0, 0, 0, 0, false};
    const uint32_t e = b + p.chunk < total ? b + p.chunk : total;
    return {b, e, p.number[b], p.number[e - 1], true};
}

// (scale: p.scale, or 0 for a row without tokens, which is to be 0 whatever p.scale is)
template <typename T>
__device__ __forceinline__ void finish_row(Sums<T> &a, const EmbedGradParams &p, const Columns<T> &c, uint32_t v, uint32_t q, float scale)
{
    const Place to = place_of(p.W, p.w.s, p.w.s.b_shift, v, q);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) a.f[u][i] *= scale;
        c.template store<false>(p.W, to, u, pack16(a.f[u], T()));
    }
}

// a run's parts of numbers with many tokens, as partial sums
template <typename T> __device__ __forceinline__ void sum_run(const EmbedGradParams &p, const WaveWork &g)
{
    if (g.row >= p.runs) return;
    const Run r = run_of(p, g.row);
    if (!r.any) return;
    const Columns<T> c(p.w.s, g.j0);
    const Sources<T> src(p, g);
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        if (side == 1 && r.last == r.first) break;
        const uint32_t at = uniform(place(p.to, side == 0 ? r.first : r.last)), vb = load_scalar(p.start + at), ve = load_scalar(p.start + at + 1);
        if (ve - vb <= p.chunk) continue; // (a number with more tokens than a run holds reaches the run's first or last place)
        Sums<T> a;
        a.clear();
        add_rows<T, kRunBatch>(a, p, src, c, vb > r.b ? vb : r.b, ve < r.e ? ve : r.e);
        float *to = partial_of(p, g.row, vb > r.b, g.q);
#pragma unroll
        for (int u = 0; u < kU; ++u)
#pragma unroll
            for (int i = 0; i < kVec<T>; i += 4)
                store16(to + c.col[u] + i, u32x4{__float_as_uint(a.f[u][i]), __float_as_uint(a.f[u][i + 1]), __float_as_uint(a.f[u][i + 2]), __float_as_uint(a.f[u][i + 3])});
    }
}

// p.rows numbers, 8 lanes to each of them: where their tokens begin comes in one load, and the first 8 tokens of each in another.
// The numbers lie p.apart from each other: the frequent ones, which neighbour each other in most vocabularies, go to
// different waves.
template <typename T> __device__ __forceinline__ void sum_rows(const EmbedGradParams &p, const WaveWork &g)
{
    const uint32_t lane = threadIdx.x & 63u, vocab = (uint32_t)p.vocab;
    const Columns<T> c(p.w.s, g.j0);
    const Sources<T> src(p, g);
    Sums<T> a;
    const uint32_t v0 = g.row;
    if (v0 >= p.apart) return;
    uint32_t begin = 0, end = 0, tokens = 0;
    {
        const uint32_t k = lane >> 3, v = v0 + k * p.apart;
        if (k < p.rows && v < vocab) {
            const uint32_t at = place(p.to, v);
            begin = p.start[at];
            end = p.start[at + 1];
            if (begin + (lane & 7u) < end) tokens = p.order[begin + (lane & 7u)];
        }
    }
#pragma unroll 1
    for (uint32_t k = 0; k < p.rows; ++k) {
        const uint32_t v = v0 + k * p.apart, b = wave::read_lane(begin, (int)k * 8), e = wave::read_lane(end, (int)k * 8);
        if (v >= vocab) break;
        if (e - b > p.chunk) continue; // (runs)
        if (e == b) { // most rows
            const Place to = place_of(p.W, p.w.s, p.w.s.b_shift, v, g.q);
#pragma unroll
            for (int u = 0; u < kU; ++u) c.template store<false>(p.W, to, u, u32x4{0, 0, 0, 0});
            continue;
        }
        a.clear();
        const uint32_t n = e - b < 8 ? e - b : 8;
        for (uint32_t i = 0; i < n; i += kRowBatch)
            add_batch<T, kRowBatch>(a, p, src, c, n - i, [&](int j) { return wave::read_lane(tokens, (int)(k * 8 + i) + j); });
        if (b + 8 < e) add_rows<T, kRowBatch>(a, p, src, c, b + 8, e);
        finish_row(a, p, c, v, g.q, p.scale);
    }
}

// The row of a number with many tokens whose first one lies in the run (there is one such number at most, the run's last): the sum
// over its partial sums.
struct Long { uint32_t v, b, last; bool any; };
__device__ __forceinline__ Long long_of(const EmbedGradParams &p, uint32_t run)
{
    const Run r = run_of(p, run);
    if (!r.any) return {0, 0, 0, false};
    const uint32_t at = place(p.to, r.last), b = p.start[at], e = p.start[at + 1];
    return {r.last, b, quotient(e - 1, p.by_chunk), b >= r.b && e - b > p.chunk};
}
// (the first of its partial sums counts as begun inside the run unless it is the run's first place)
__device__ __forceinline__ const float *partial_in(const EmbedGradParams &p, uint32_t run, uint32_t first_run, bool inside, uint32_t q)
{
    return partial_of(p, run, run == first_run && inside, q);
}

template <typename T> __device__ __forceinline__ void join_runs(const EmbedGradParams &p, const WaveWork &g)
{
    if (g.row >= p.runs) return;
    const Long w = long_of(p, g.row);
    if (!w.any) return;
    const uint32_t v = uniform(w.v), last = uniform(w.last);
    const bool inside = uniform(w.b) > g.row * p.chunk;
    const Columns<T> c(p.w.s, g.j0);
    Sums<T> a;
    a.clear();
    for (uint32_t run = g.row; run <= last; run += kPartials) {
        u32x4 r[kPartials][kU][kVec<T> / 4];
#pragma unroll
        for (int k = 0; k < kPartials; ++k) {
            if (run + k > last) break;
            const float *from = partial_in(p, run + k, g.row, inside, g.q);
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int i = 0; i < kVec<T> / 4; ++i) r[k][u][i] = load16(from + c.col[u] + 4 * i);
        }
#pragma unroll
        for (int k = 0; k < kPartials; ++k) {
            if (run + k > last) break;
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int i = 0; i < kVec<T>; ++i) a.f[u][i] += __uint_as_float(r[k][u][i / 4][i % 4]);
        }
    }
    finish_row(a, p, c, v, g.q, p.scale);
}

// (2) The first workgroups' waves take a run each, beside the rows.  (The runs in a launch of their own in front, and the joins in
// this one: 2 to 3 % faster at 65536 x 8192 and 16384 tokens, 10 % slower at 32000 x 1024 and 8192.)
template <typename T> __global__ __launch_bounds__(kThreads) void embed_sums_wide_kernel(const EmbedGradParams p)
{
    if (blockIdx.x < p.run_groups) sum_run<T>(p, wave_work(p.w, blockIdx.x));
    else sum_rows<T>(p, wave_work(p.w, blockIdx.x - p.run_groups));
}
// (3)
template <typename T> __global__ __launch_bounds__(kThreads) void embed_join_wide_kernel(const EmbedGradParams p)
{
    join_runs<T>(p, wave_work(p.w, blockIdx.x));
}

// the rows of places [b, e) of the sorted list, a vector of each, kRunBatch of them on their way together
template <typename T>
__device__ __forceinline__ void add_vectors(float (&s)[kVec<T>], const EmbedGradParams &p, const LaneWork &g, const Small<T> &c, uint32_t b, uint32_t e)
{
    for (uint32_t i = b; i < e; i += kRunBatch) {
        uint32_t t[kRunBatch];
        u32x4 r[kRunBatch];
#pragma unroll
        for (int k = 0; k < kRunBatch; ++k) t[k] = p.order[i + k < e ? i + k : e - 1];
#pragma unroll
        for (int k = 0; k < kRunBatch; ++k) r[k] = c.load(source_of<T>(p.G, p.w.s, p.w.s.a_shift, t[k], g.q));
#pragma unroll
        for (int k = 0; k < kRunBatch; ++k) {
            float f[kVec<T>];
            unpack16(r[k], f, T());
#pragma unroll
            for (int q = 0; q < kVec<T>; ++q) s[q] = i + k < e ? s[q] + f[q] : s[q];
        }
    }
}
template <typename T, class C>
__device__ __forceinline__ void finish_vector(float (&s)[kVec<T>], const EmbedGradParams &p, const LaneWork &g, const C &c, uint32_t v, float scale)
{
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) s[i] *= scale;
    c.store(p.W, place_of(p.W, p.w.s, p.w.s.b_shift, v, g.q), pack16(s, T()));
}

template <typename T> __global__ __launch_bounds__(kThreads) void embed_sums_narrow_kernel(const EmbedGradParams p)
{
    const LaneWork g = small_work(p.w);
    const Small<T> c(p.w.s);
    if (g.row < p.runs) {
        const Run r = run_of(p, g.row);
        if (!r.any) return;
        for (int side = 0; side < 2; ++side) {
            if (side == 1 && r.last == r.first) break;
            const uint32_t at = place(p.to, side == 0 ? r.first : r.last), vb = p.start[at], ve = p.start[at + 1];
            if (ve - vb <= p.chunk) continue;
            float s[kVec<T>] = {};
            add_vectors<T>(s, p, g, c, vb > r.b ? vb : r.b, ve < r.e ? ve : r.e);
            c.store_floats(s, partial_of(p, g.row, vb > r.b, g.q));
        }
        return;
    }
    const uint32_t v = g.row - p.runs;
    if ((int64_t)v >= p.vocab) return;
    const uint32_t at = place(p.to, v), b = p.start[at], e = p.start[at + 1];
    if (e - b > p.chunk) return; // (runs)
    float s[kVec<T>] = {};
    add_vectors<T>(s, p, g, c, b, e);
    finish_vector<T>(s, p, g, c, v, b < e ? p.scale : 0.0f);
}

template <typename T> __global__ __launch_bounds__(kThreads) void embed_join_narrow_kernel(const EmbedGradParams p)
{
    const LaneWork g = small_work(p.w);
    const Small<T> c(p.w.s);
    if (g.row >= p.runs) return;
    const Long w = long_of(p, g.row);
    if (!w.any) return;
    const bool inside = w.b > g.row * p.chunk;
    float s[kVec<T>] = {};
    for (uint32_t run = g.row; run <= w.last; run += kPartials) {
        float f[kPartials][kVec<T>];
#pragma unroll
        for (int k = 0; k < kPartials; ++k) c.load_floats(f[k], partial_in(p, run + k < w.last ? run + k : w.last, g.row, inside, g.q));
#pragma unroll
        for (int k = 0; k < kPartials; ++k)
#pragma unroll
            for (int i = 0; i < kVec<T>; ++i) s[i] = run + k <= w.last ? s[i] + f[k][i] : s[i];
    }
    finish_vector<T>(s, p, g, c, w.v, p.scale);
}

// Few tokens: nothing to sort.  Every wave holds all token numbers, 64 to a register, and asks for each of its rows which of them
// are the row's; one launch.  With / without, us: 50000 x 1024 from 16 tokens 19 / 23 (5.4 TB/s), from 256 19 / 25, 1000 x 4096 from
// 256 12 / 17.
constexpr uint32_t kFewTokens = 256, kFewRegisters = kFewTokens / 64;
struct Found {
    uint64_t in[kFewRegisters];
    __device__ __forceinline__ bool any() const
    {
        uint64_t m = 0;
#pragma unroll
        for (uint32_t i = 0; i < kFewRegisters; ++i) m |= in[i];
        return m != 0;
    }
    // takes out the first one
    __device__ __forceinline__ uint32_t next()
    {
        uint32_t t = 0;
        bool done = false;
#pragma unroll
        for (uint32_t i = 0; i < kFewRegisters; ++i) {
            if (done || in[i] == 0) continue;
            t = i * 64 + (uint32_t)__builtin_ctzll(in[i]);
            in[i] &= in[i] - 1;
            done = true;
        }
        return t;
    }
};
template <typename I> struct Few {
    uint32_t number[kFewRegisters];
    __device__ __forceinline__ Few(const EmbedGradParams &p)
    {
#pragma unroll
        for (uint32_t i = 0; i < kFewRegisters; ++i) {
            const uint32_t t = i * 64 + (threadIdx.x & 63u);
            const int64_t v = p.tokens ? token_at<I>(p.ids, t < p.tokens ? t : p.tokens - 1) : -1;
            number[i] = t < p.tokens && v >= 0 && v < p.vocab ? (uint32_t)v : kNoToken;
        }
    }
    // the tokens with numbers in [v, v + n)
    __device__ __forceinline__ Found of(uint32_t v, uint32_t n) const
    {
        Found f;
#pragma unroll
        for (uint32_t i = 0; i < kFewRegisters; ++i) f.in[i] = wave::ballot(number[i] != kNoToken && number[i] - v < n);
        return f;
    }
    __device__ __forceinline__ uint32_t number_of(uint32_t t) const
    {
        uint32_t v = 0;
#pragma unroll
        for (uint32_t i = 0; i < kFewRegisters; ++i)
            if (t / 64 == i) v = wave::read_lane(number[i], (int)(t & 63u));
        return v;
    }
};

template <typename T, typename I> __global__ __launch_bounds__(kThreads) void embed_few_wide_kernel(const EmbedGradParams p)
{
    const WaveWork g = wave_work(p.w, blockIdx.x);
    if (g.row >= p.apart) return;
    const Few<I> few(p);
    const Columns<T> c(p.w.s, g.j0);
    const Sources<T> src(p, g);
#pragma unroll 1
    for (uint32_t k = 0; k < p.rows; ++k) {
        const uint32_t v = g.row + k * p.apart;
        if (v >= (uint32_t)p.vocab) break;
        Found f = few.of(v, 1);
        const float scale = f.any() ? p.scale : 0.0f;
        Sums<T> a;
        a.clear();
        while (f.any()) {
            uint32_t t[kRowBatch], n = 0;
#pragma unroll
            for (int i = 0; i < kRowBatch; ++i) {
                n += f.any() ? 1 : 0;
                t[i] = f.next();
            }
            add_batch<T, kRowBatch>(a, p, src, c, n, [&](int i) { return t[i]; });
        }
        finish_row(a, p, c, v, g.q, scale);
    }
}

template <typename T, typename I> __global__ __launch_bounds__(kThreads) void embed_few_narrow_kernel(const EmbedGradParams p)
{
    const LaneWork g = lane_work(p.w);
    const Column1<T> c(p.w.s, g.j);
    const Few<I> few(p);
    // the wave's rows: those of its first and its last lane, and what lies between
    const uint32_t v0 = wave::read_lane(g.row, 0), v1 = wave::read_lane(g.row, 63);
    Found f = few.of(v0, v1 - v0 + 1);
    float s[kVec<T>] = {}, scale = 0.0f;
    while (f.any()) {
        uint32_t t[kRowBatch], v[kRowBatch], m = 0;
        u32x4 r[kRowBatch];
#pragma unroll
        for (int i = 0; i < kRowBatch; ++i) {
            m += f.any() ? 1 : 0;
            t[i] = f.next();
            v[i] = few.number_of(t[i]);
            r[i] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < kRowBatch; ++i)
            if ((uint32_t)i < m && v[i] == g.row && c.own) r[i] = c.load(source_of<T>(p.G, p.w.s, p.w.s.a_shift, t[i], g.q));
#pragma unroll
        for (int i = 0; i < kRowBatch; ++i) {
            if ((uint32_t)i >= m || v[i] != g.row) continue;
            scale = p.scale;
            float x[kVec<T>];
            unpack16(r[i], x, T());
#pragma unroll
            for (int q = 0; q < kVec<T>; ++q) s[q] += x[q];
        }
    }
    if (g.row < (uint32_t)p.vocab) finish_vector<T>(s, p, g, c, g.row, scale);
}

// ----------------------------------------------------------------------------------------------------- host side

tt_status check_sizes(int64_t tokens, int64_t vocab, int64_t width, int k, int dtype, const tt_tiling &a, const tt_tiling &b)
{
    if (!valid_k(k) || !valid_tiling(a, k) || !valid_tiling(b, k) || !valid_dtype(dtype)) return TT_EINVAL;
    if (tokens < 0 || vocab < 0 || width < 0) return TT_EINVAL;
    if (!fits31(tokens) || vocab >= (int64_t(1) << 30) || !fits31(width)) return TT_EUNSUPPORTED;
    return TT_OK;
}

bool valid_ids(int id_dtype, const void *ids, int64_t tokens)
{
    if (id_dtype != TT_I32 && id_dtype != TT_I64) return false;
    return tokens == 0 || aligned_to(ids, id_dtype == TT_I32 ? 4 : 8);
}

// Places of the sorted list per run: a run is added up by one wave and the runs of a number by another, so both are to stay short.
// 8000 x 4096 from 16384 tokens, runs of 32 / 64, us: 70 / 72 (65536 x 8192: 298 / 291); from 32768, runs of 32 / 64 / 128: 114 / 107 / 115.
uint32_t run_length(int64_t tokens) { return tokens <= 16384 ? 32 : tokens <= 65536 ? 64 : 128; }

// the numbers' places: 256 workgroups, one a CU, or as many as make a workgroup's counters enough
Places places_of(int64_t vocab)
{
    Places s{0, 0};
    while (s.wlog < 8 && (int64_t(1) << s.wlog) < vocab) ++s.wlog;
    while (((vocab + (int64_t(1) << s.wlog) - 1) >> s.wlog) > kSortRange) ++s.wlog;
    s.range = (uint32_t)((vocab + (int64_t(1) << s.wlog) - 1) >> s.wlog);
    return s;
}

struct GradSpace {
    size_t order, number, start, partial, bytes;
    uint32_t runs;
    Places to;
};
GradSpace grad_space(int64_t tokens, int64_t vocab, int64_t width)
{
    GradSpace s{0, 0, 0, 0, 0, 0, places_of(vocab)};
    if (tokens <= (int64_t)kFewTokens) return s; // (nothing is sorted)
    const uint32_t chunk = run_length(tokens);
    s.runs = tokens > chunk ? (uint32_t)((tokens + chunk - 1) / chunk) : 0;
    s.number = align_up((size_t)tokens * 4, 256);
    s.start = 2 * s.number;
    s.partial = s.start + align_up((((size_t)s.to.range << s.to.wlog) + 1) * 4, 256);
    s.bytes = s.partial + align_up((size_t)2 * s.runs * (size_t)width * 4, 256);
    return s;
}

// What covers any smaller number of tokens too: the runs are as many as ever in front of where they get longer.
size_t grad_room(int64_t tokens, int64_t vocab, int64_t width)
{
    size_t room = 0;
    for (int64_t t : {(int64_t)16384, (int64_t)65536, tokens})
        if (t <= tokens) room = std::max(room, grad_space(t, vocab, width).bytes);
    return room;
}

tt_status launched() { return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE; }

template <typename T, typename I> tt_status launch_embed(const EmbedParams &p, uint32_t grid, hipStream_t s)
{
    if (p.w.wide) hipLaunchKernelGGL((embed_wide_kernel<T, I>), dim3(grid), dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((embed_narrow_kernel<T, I>), dim3(grid), dim3(kThreads), 0, s, p);
    return launched();
}

} // namespace
} // namespace tt

extern "C" tt_status tt_embed_forward(int64_t tokens, int64_t vocab, int64_t width, int k, int dtype, tt_tiling tW, tt_tiling tX,
                                      int id_dtype, const void *ids, float scale, const void *const *W, void *const *X,
                                      void *stream)
{
    using namespace tt;
    tt_status st = check_sizes(tokens, vocab, width, k, dtype, tW, tX);
    if (st != TT_OK) return st;
    const int e = dtype_bytes(dtype);
    if (!valid_ids(id_dtype, ids, tokens) || !shards_fit(W, k, e, vocab == 0 || width == 0) ||
        !shards_fit(const_cast<const void *const *>(X), k, e, tokens == 0 || width == 0))
        return TT_EINVAL;
    EmbedParams p;
    if (!make_blocks(W, tW, k, vocab, width, &p.W) || !make_blocks(const_cast<const void *const *>(X), tX, k, tokens, width, &p.X)) return TT_EINFEASIBLE;
    if (tokens == 0 || width == 0) return TT_OK;
    p.w = split_rows(p.W, p.X, width, 16 / e, false);
    p.ids = ids;
    p.tokens = (uint32_t)tokens;
    p.vocab = vocab;
    p.scale = scale;
    const uint64_t grid = groups_of(p.w, (uint64_t)tokens);
    if (grid * kThreads >= (uint64_t(1) << 31)) return TT_EUNSUPPORTED;
    const uint64_t row = (uint64_t)width * e;
    ProfileScope scope(stream, TT_K_EMBED, 1 << k, tokens, width, e, (uint64_t)tokens * row * (1 + p.X.nrep), 0);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (dtype == TT_BF16) return id_dtype == TT_I32 ? launch_embed<uint16_t, int32_t>(p, (uint32_t)grid, s) : launch_embed<uint16_t, int64_t>(p, (uint32_t)grid, s);
    return id_dtype == TT_I32 ? launch_embed<float, int32_t>(p, (uint32_t)grid, s) : launch_embed<float, int64_t>(p, (uint32_t)grid, s);
}

extern "C" tt_status tt_embed_workspace_bytes(int64_t tokens, int64_t vocab, int64_t width, int k, int dtype, tt_tiling tdX,
                                              tt_tiling tdW, size_t *bytes)
{
    using namespace tt;
    if (!bytes) return TT_EINVAL;
    tt_status st = check_sizes(tokens, vocab, width, k, dtype, tdX, tdW);
    if (st != TT_OK) return st;
    Grid g;
    if (!make_grid(tdX.cut, k, tokens, width, &g) || !make_grid(tdW.cut, k, vocab, width, &g)) return TT_EINFEASIBLE;
    *bytes = grad_room(tokens, vocab, width);
    return TT_OK;
}

namespace tt {
namespace {

template <typename T, typename I>
tt_status launch_embed_grad(const SortParams &sp, const EmbedGradParams &p, uint32_t run_groups, uint32_t row_groups, hipStream_t s)
{
    if (p.tokens <= kFewTokens) {
        if (p.w.wide) hipLaunchKernelGGL((embed_few_wide_kernel<T, I>), dim3(row_groups), dim3(kThreads), 0, s, p);
        else hipLaunchKernelGGL((embed_few_narrow_kernel<T, I>), dim3(row_groups), dim3(kThreads), 0, s, p);
        return launched();
    }
    hipLaunchKernelGGL((sort_tokens_kernel<I>), dim3(1u << sp.to.wlog), dim3(kSortThreads), 0, s, sp);
    if (p.w.wide) {
        hipLaunchKernelGGL((embed_sums_wide_kernel<T>), dim3(row_groups), dim3(kThreads), 0, s, p);
        if (run_groups) hipLaunchKernelGGL((embed_join_wide_kernel<T>), dim3(run_groups), dim3(kThreads), 0, s, p);
    } else {
        hipLaunchKernelGGL((embed_sums_narrow_kernel<T>), dim3(row_groups), dim3(kThreads), 0, s, p);
        if (run_groups) hipLaunchKernelGGL((embed_join_narrow_kernel<T>), dim3(run_groups), dim3(kThreads), 0, s, p);
    }
    return launched();
}

} // namespace
} // namespace tt

extern "C" tt_status tt_embed_backward(int64_t tokens, int64_t vocab, int64_t width, int k, int dtype, tt_tiling tdX, tt_tiling tdW,
                                       int id_dtype, const void *ids, float scale, const void *const *dX, void *const *dW,
                                       void *workspace, size_t ws_bytes, void *stream)
{
    using namespace tt;
    tt_status st = check_sizes(tokens, vocab, width, k, dtype, tdX, tdW);
    if (st != TT_OK) return st;
    const int e = dtype_bytes(dtype);
    if (!valid_ids(id_dtype, ids, tokens) || !shards_fit(dX, k, e, tokens == 0 || width == 0) ||
        !shards_fit(const_cast<const void *const *>(dW), k, e, vocab == 0 || width == 0))
        return TT_EINVAL;
    EmbedGradParams p;
    if (!make_blocks(dX, tdX, k, tokens, width, &p.G) || !make_blocks(const_cast<const void *const *>(dW), tdW, k, vocab, width, &p.W)) return TT_EINFEASIBLE;
    if (vocab == 0 || width == 0) return TT_OK;
    const GradSpace sp = grad_space(tokens, vocab, width);
    if (sp.bytes && (!workspace || ws_bytes < sp.bytes || reinterpret_cast<uintptr_t>(workspace) % 256)) return TT_EWORKSPACE;
    char *ws = static_cast<char *>(workspace);
    SortParams q;
    q.ids = ids;
    q.tokens = (uint32_t)tokens;
    q.vocab = vocab;
    q.to = sp.to;
    q.order = reinterpret_cast<uint32_t *>(ws + sp.order);
    q.number = reinterpret_cast<uint32_t *>(ws + sp.number);
    q.start = reinterpret_cast<uint32_t *>(ws + sp.start);
    p.w = split_rows(p.G, p.W, width, 16 / e, tokens <= (int64_t)kFewTokens);
    p.ids = ids;
    p.order = q.order;
    p.number = q.number;
    p.start = q.start;
    p.partial = reinterpret_cast<float *>(ws + sp.partial);
    p.to = sp.to;
    p.places = sp.to.range << sp.to.wlog;
    p.tokens = (uint32_t)tokens;
    p.chunk = run_length(tokens);
    p.by_chunk = divisor(p.chunk);
    p.runs = sp.runs;
    p.cols = (uint32_t)width;
    p.vocab = vocab;
    p.scale = scale;
    // Rows per wave: as many as leave every CU 32 waves, 4 at most (65536 x 8192, us with 2, 4, 8 of them:
    // no tokens 178, 190, 192; 16384 tokens 301, 295, 297), 2 where there is nothing to look up first.
    const uint64_t waves = (uint64_t)vocab * p.w.s.nseg * p.w.parts;
    const uint32_t most = tokens <= (int64_t)kFewTokens ? 2 : 4;
    p.rows = most == 4 && waves >= 4 * 8192 ? 4 : waves >= 2 * 8192 ? 2 : 1;
    p.apart = (uint32_t)((vocab + p.rows - 1) / p.rows);
    const uint64_t run_groups = groups_of(p.w, sp.runs), row_groups = p.w.wide ? run_groups + groups_of(p.w, p.apart) : groups_of(p.w, (uint64_t)sp.runs + (uint64_t)vocab);
    if (run_groups * kThreads >= (uint64_t(1) << 31) || row_groups * kThreads >= (uint64_t(1) << 31)) return TT_EUNSUPPORTED;
    const uint64_t row = (uint64_t)width * e;
    ProfileScope scope(stream, TT_K_EMBED_GRAD, 1 << k, vocab, width, e, (uint64_t)tokens * row + (uint64_t)vocab * row * p.W.nrep, 0);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const uint32_t rg = (uint32_t)run_groups, wg = (uint32_t)row_groups;
    p.run_groups = p.w.wide ? rg : 0;
    if (dtype == TT_BF16)
        return id_dtype == TT_I32 ? launch_embed_grad<uint16_t, int32_t>(q, p, rg, wg, s)
                                  : launch_embed_grad<uint16_t, int64_t>(q, p, rg, wg, s);
    return id_dtype == TT_I32 ? launch_embed_grad<float, int32_t>(q, p, rg, wg, s)
                              : launch_embed_grad<float, int64_t>(q, p, rg, wg, s);
}
