// How kernels walk over the rows of tiled tensors with a row in registers: which lanes hold what of it, loads, stores, and sums and
// maxima over it.
//
//   GroupWalk   rows of up to 32 vectors, of up to 64 in several segments, and of segments of less than a vector: a power of two of
//               lanes a row, a vector each
//   SlotWalk    others: one wave or several a row.  A segment (row_walk.h) is dealt out in slots of 64 vectors, so that what a wave loads
//               at a time lies in one block: row, block and address are scalars, and a lane adds its place in the slot.
#pragma once
#include "row_walk.h"

namespace tt {

constexpr int kCUs = 256;                // of an MI355X
constexpr uint32_t kWaveBlock = 256;     // threads of a workgroup whose waves hold a row or several each
constexpr uint32_t kMostThreads = 1024;  // ... of one that holds a row
constexpr int kMostWaves = kMostThreads / 64;

__device__ __forceinline__ float lane_xor(float v, uint32_t m) { return __uint_as_float(wave::shfl_xor(__float_as_uint(v), (int)m)); }
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, uint32_t m) { return wave::shfl_xor(v, (int)m); }
__device__ __forceinline__ double lane_xor(double v, uint32_t m) { return wave::shfl_xor(v, (int)m); }

struct Sum {
    template <typename V> static __device__ __forceinline__ V of(V a, V b) { return a + b; }
    static __device__ __forceinline__ float over_wave(float v) { return wave_sum(v); }
};
// ... of fp32 values that travel as their bits
struct SumBits {
    static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }
    static __device__ __forceinline__ uint32_t over_wave(uint32_t v) { return __float_as_uint(wave_sum(__uint_as_float(v))); }
};
// The largest of values that are not negative, by their bits: an infinity is above every number and a NaN above that.
struct Largest {
    static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; }
    static __device__ __forceinline__ uint32_t over_wave(uint32_t v) { return wave::combined(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
    static __device__ __forceinline__ double of(double a, double b)
    {
        return __builtin_bit_cast(uint64_t, a) > __builtin_bit_cast(uint64_t, b) ? a : b;
    }
};

// v combined over `lanes` neighbouring lanes (a power of two)
template <class F, typename V> __device__ __forceinline__ V over_lanes(V v, uint32_t lanes)
{
    if constexpr (sizeof(V) == 4) {
        if (lanes == 64) return F::over_wave(v);
    }
    for (uint32_t m = 1; m < lanes; m <<= 1) v = F::of(v, lane_xor(v, m));
    return v;
}

// LDS of the reductions over several waves.  Two sets in turn, so that one barrier a reduction is enough: a set is written again only
// after the barrier of the reduction between, which all threads pass after they have read it.
template <int N> struct RowScratch { double v[2][N][kMostWaves]; };

// N values at a time combined over the waves of a workgroup, value i by F[i]; `turn` alternates from call to call.
template <typename V, class... F, class S> __device__ __forceinline__ void over_workgroup(V (&v)[sizeof...(F)], uint32_t waves, S &scratch, uint32_t turn)
{
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int i = 0;
    ((v[i] = over_lanes<F>(v[i], 64u), ++i), ...);
    if (waves == 1) return;
    if (lane == 0) {
        for (i = 0; i < (int)sizeof...(F); ++i) reinterpret_cast<V *>(scratch.v[turn & 1][i])[wave] = v[i];
    }
    __syncthreads();
    i = 0;
    // (16 waves at most: the lanes behind them have nothing to add)
    ((v[i] = over_lanes<F>(lane < waves ? reinterpret_cast<const V *>(scratch.v[turn & 1][i])[lane] : V(0), 64u), ++i), ...);
}

// How a launch lays its rows out
enum RowKind { kGroups, kSlots, kLong };
struct RowLaunch {
    RowKind kind;
    int vectors;          // of a lane
    uint32_t lanes;       // kGroups: of a row
    uint32_t waves;       // kSlots: of a row
    uint32_t block;       // threads of a workgroup
    uint32_t at_once;     // rows of a workgroup at a time
};

struct RowWalk {
    RowShape r;
    uint32_t slots_per_seg, slots;
    Divisor by_slots; // slots of a segment
    uint32_t rows, groups, lanes, waves;
    uint32_t once;  // results are stored past the caches
    uint32_t flags; // of the kernel
};

// Results that the caches do not hold until they are read, all of a call's together, are stored past them: 16384 x 4096 bf16 sum and norm
// 106 -> 101 us, gradients of 16384 x 8192 over 8 shards 294 -> 280.
constexpr uint64_t kOnceBytes = uint64_t(64) << 20;

inline RowWalk row_walk(const BlockTable &a, const BlockTable &b, int64_t rows, int64_t cols, int ev)
{
    RowWalk w;
    w.r = row_shape(a, b, cols, ev);
    w.slots_per_seg = (w.r.s.vps + 63) / 64;
    w.slots = w.r.s.nseg * w.slots_per_seg;
    w.by_slots = divisor(w.slots_per_seg);
    w.rows = (uint32_t)rows;
    w.groups = w.lanes = w.waves = w.once = w.flags = 0;
    return w;
}
// most: vectors of a lane where that is enough for the row;  limit: where it is not
inline RowLaunch row_launch(RowWalk *w, int ev, uint32_t most = 4, uint32_t limit = 4)
{
    RowLaunch l{kLong, 0, 64, kMostWaves, kMostThreads, 1};
    // rows of up to 32 vectors, or 64 in segments that would leave half of the slots empty (a row of narrow segments has at most 64)
    if (w->r.units <= 32 || (w->r.units <= 64 && w->slots > 1) || narrow_segments(w->r, ev)) {
        uint32_t lanes = 1;
        while (lanes < w->r.units) lanes <<= 1;
        l = {kGroups, 1, lanes, 0, kWaveBlock, kWaveBlock / lanes};
    } else {
        // Several vectors a lane where there are waves enough all the same: the sums of a row, its addresses and its barrier are paid by
        // the wave.  Sum and norm of 16384 rows of 2048 bf16 with one a lane 53.4 us, two 51.9, four 48.7; of 4096 105, 103, 102.
        uint32_t best = ~0u;
        for (uint32_t v = 1; v <= (best == ~0u ? limit : most); ++v) {
            const uint32_t waves = (w->slots + v - 1) / v, cost = 10 * waves * v + 7 * waves;
            if (waves > (uint32_t)kMostWaves || (best != ~0u && (uint64_t)w->rows * waves < 16 * kCUs) || cost >= best) continue;
            best = cost;
            l = {kSlots, (int)v, 64, waves, waves == 1 ? kWaveBlock : waves * 64, waves == 1 ? kWaveBlock / 64 : 1};
        }
    }
    w->lanes = l.lanes;
    w->waves = l.waves;
    return l;
}
// workgroups of a launch whose workgroups walk over rows: what the CUs hold at a time, of so many threads each
inline uint32_t row_groups(const RowLaunch &l, int64_t rows, uint32_t threads = 2048)
{
    const int64_t all = (rows + l.at_once - 1) / l.at_once, held = (int64_t)kCUs * (threads / l.block);
    return (uint32_t)(all < held ? all : held);
}

// kinds of memory access
enum { kPlain = 0, kCut = 1, kNarrow = 2 };

// The walks.  V vectors a lane: vector i is spot(i) of row(base), `base` from first() on in steps of step().  A: whether a tensor is of
// the first grid or of the second.
template <typename T, int MODE> struct GroupWalk {
    static constexpr int V = 1;
    static constexpr uint32_t EV = kVec<T>;
    static constexpr bool CUT = MODE != kPlain, NARROW = MODE == kNarrow;
    Spot v;
    __device__ __forceinline__ void init(const RowWalk &w) { v = spot_of<EV>(w.r, threadIdx.x & (w.lanes - 1)); }
    __device__ __forceinline__ uint32_t at_once(const RowWalk &w) const { return kWaveBlock / w.lanes; }
    __device__ __forceinline__ uint32_t row(const RowWalk &w, uint32_t base) const { return base + threadIdx.x / w.lanes; }
    // this lane's number among those of the row
    __device__ __forceinline__ uint32_t number(const RowWalk &w) const { return threadIdx.x & (w.lanes - 1); }
    __device__ __forceinline__ uint32_t count(const RowWalk &w) const { return w.lanes; }
    __device__ __forceinline__ uint32_t column(const RowWalk &w, int) const { return v.q * w.r.s.seg + v.at; }
    __device__ __forceinline__ Spot spot(const RowWalk &, int) const { return v; }
    // the vector without the leading values that another lane counts
    __device__ __forceinline__ u32x4 counted(const RowWalk &, int, u32x4 x) const { return v.dup ? without(x, v.dup, T()) : x; }
    // where the row's vector i lies in a grid (the same for all tensors of the grid)
    template <bool A> __device__ __forceinline__ Place place(const RowWalk &w, const BlockTable &b, uint32_t row, int) const
    {
        const Lane l = lane_of<CUT>(b, w.r.s, A ? w.r.s.a_shift : w.r.s.b_shift, row, v);
        return {l.block, l.at};
    }
    __device__ __forceinline__ u32x4 load(const BlockTable &b, const Place &p, const Spot &) const { return load_spot<T, NARROW>(b, {p.block, p.at}, v); }
    // (once: nobody reads it soon)
    __device__ __forceinline__ void store(const BlockTable &b, const Place &p, const Spot &, u32x4 x, bool once) const
    {
        store_spot<T, CUT, NARROW>(b, {p.block, p.at}, v, x, once);
    }
    __device__ __forceinline__ u32x4 by_column(const RowWalk &w, const void *p, int i) const
    {
        const T *g = static_cast<const T *>(p) + column(w, i);
        if constexpr (NARROW) return load_part(g, v.n);
        else return load16(g);
    }
    template <typename X, class... F, class S> __device__ __forceinline__ void reduce(const RowWalk &w, X (&x)[sizeof...(F)], S &, uint32_t) const
    {
        int i = 0;
        ((x[i] = over_lanes<F>(x[i], w.lanes), ++i), ...);
    }
    static __device__ __forceinline__ bool any(bool p) { return wave::ballot(p) != 0; } // of the wave's rows
    static __device__ __forceinline__ u32x4 without(u32x4 x, uint32_t n, uint16_t)
    {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) x[i] = n >= 2 * i + 2 ? 0u : n == 2 * i + 1 ? x[i] & 0xffff0000u : x[i];
        return x;
    }
    static __device__ __forceinline__ u32x4 without(u32x4 x, uint32_t n, float)
    {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) x[i] = n > i ? 0u : x[i];
        return x;
    }
};

template <typename T, int NV, bool CUTS> struct SlotWalk {
    static constexpr int V = NV;
    static constexpr bool CUT = CUTS, NARROW = false;
    static constexpr uint32_t EV = kVec<T>;
    uint32_t wave; // of the row
    __device__ __forceinline__ void init(const RowWalk &w) { wave = w.waves == 1 ? 0u : uniform(threadIdx.x >> 6); }
    __device__ __forceinline__ uint32_t at_once(const RowWalk &w) const { return w.waves == 1 ? kWaveBlock / 64 : 1; }
    __device__ __forceinline__ uint32_t row(const RowWalk &w, uint32_t base) const { return w.waves == 1 ? base + uniform(threadIdx.x >> 6) : base; }
    __device__ __forceinline__ uint32_t number(const RowWalk &w) const { return w.waves == 1 ? threadIdx.x & 63 : threadIdx.x; }
    __device__ __forceinline__ uint32_t count(const RowWalk &w) const { return w.waves * 64; }
    // slot i of the wave: segment, and its first vector there (worked out where it is used: kept for all slots they leave no scalar registers)
    struct Slot { uint32_t q, first; };
    __device__ __forceinline__ Slot slot(const RowWalk &w, int i) const
    {
        uint32_t s = wave + i * w.waves;
        wave::forget_uniform(s);
        if constexpr (!CUT) return {0, s * 64};
        const uint32_t q = quotient(s, w.by_slots);
        return {q, (s - q * w.slots_per_seg) * 64};
    }
    // all of its lanes have a vector of their own
    __device__ __forceinline__ bool whole(const RowWalk &w, const Slot &s) const
    {
        return (!CUT || s.q < w.r.s.nseg) && s.first + 64 + (w.r.s.tail ? 1 : 0) <= w.r.s.vps;
    }
    // (segments have a vector at least: the one that ends with the segment is the last one, and stands in for those past the end)
    __device__ __forceinline__ Spot spot(const RowWalk &w, int i) const
    {
        const Slot s = slot(w, i);
        const uint32_t j = s.first + (threadIdx.x & 63), last = w.r.s.seg - EV, q = !CUT || s.q < w.r.s.nseg ? s.q : w.r.s.nseg - 1;
        const bool there = q == s.q && j < w.r.s.vps;
        return {q, there && j * EV < last ? j * EV : last, EV, !there ? EV : j + 1 == w.r.s.vps && w.r.s.tail ? EV - w.r.s.tail : 0u};
    }
    __device__ __forceinline__ uint32_t column(const RowWalk &w, int i) const
    {
        const Spot v = spot(w, i);
        return v.q * w.r.s.seg + v.at;
    }
    __device__ __forceinline__ u32x4 counted(const RowWalk &w, int i, u32x4 x) const
    {
        if (whole(w, slot(w, i))) return x;
        return GroupWalk<T, kPlain>::without(x, spot(w, i).dup, T());
    }
    // where the slot's segment begins in the row: scalars
    template <bool A> __device__ __forceinline__ Place place(const RowWalk &w, const BlockTable &b, uint32_t row, int i) const
    {
        if constexpr (CUT) {
            const Slot s = slot(w, i);
            return place_of(b, w.r.s, A ? w.r.s.a_shift : w.r.s.b_shift, row, s.q < w.r.s.nseg ? s.q : w.r.s.nseg - 1);
        } else {
            return {0, (size_t)row * b.scols};
        }
    }
    __device__ __forceinline__ u32x4 load(const BlockTable &b, const Place &p, const Spot &v) const { return load16(static_cast<const T *>(b.p[p.block]) + p.at + v.at); }
    __device__ __forceinline__ void store(const BlockTable &b, const Place &p, const Spot &v, u32x4 x, bool once) const
    {
        store_spot<T, CUT, false>(b, {p.block, p.at + v.at}, v, x, once);
    }
    __device__ __forceinline__ u32x4 by_column(const RowWalk &w, const void *p, int i) const { return load16(static_cast<const T *>(p) + column(w, i)); }
    template <typename X, class... F, class S> __device__ __forceinline__ void reduce(const RowWalk &w, X (&x)[sizeof...(F)], S &scratch, uint32_t turn) const
    {
        over_workgroup<X, F...>(x, w.waves, scratch, turn);
    }
    // (a wave's lanes, and a workgroup's that have one row, agree)
    static __device__ __forceinline__ bool any(bool p) { return uniform((uint32_t)p) != 0; }
};

template <typename T> __device__ __forceinline__ u32x4 ones()
{
    return sizeof(T) == 2 ? u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u} : u32x4{0x3f800000u, 0x3f800000u, 0x3f800000u, 0x3f800000u};
}

// What a call has beside what every call has, as a kernel knows it: from its template argument, so that the compiler can count the
// loads and stores between a load and the wait for it (a wait that counts on fewer of them than there are waits for stores as well),
// or, for short rows, from its parameters.
constexpr int kAsGiven = -1;
template <int FLAGS> __device__ __forceinline__ bool has(uint32_t given, uint32_t flag) { return FLAGS == kAsGiven ? (given & flag) != 0 : ((uint32_t)FLAGS & flag) != 0; }

// f.run<Walk, most threads of its workgroups>() with the walk of a launch; false: rows that registers do not hold.  LIMIT as in row_launch.
template <typename T, int LIMIT = 4, class F> bool with_walk(const RowWalk &w, const RowLaunch &l, bool cut, F &&f)
{
    if (l.kind == kGroups) {
        if (narrow_segments(w.r, kVec<T>)) f.template run<GroupWalk<T, kNarrow>, kWaveBlock>();
        else if (cut) f.template run<GroupWalk<T, kCut>, kWaveBlock>();
        else f.template run<GroupWalk<T, kPlain>, kWaveBlock>();
        return true;
    }
    if (l.kind == kLong) return false;
    switch (l.vectors * 2 + cut) {
    case 2: f.template run<SlotWalk<T, 1, false>, kMostThreads>(); break;
    case 3: f.template run<SlotWalk<T, 1, true>, kMostThreads>(); break;
    case 4: f.template run<SlotWalk<T, 2, false>, kMostThreads>(); break;
    case 5: f.template run<SlotWalk<T, 2, true>, kMostThreads>(); break;
    case 6: f.template run<SlotWalk<T, 3, false>, kMostThreads>(); break;
    case 7: f.template run<SlotWalk<T, 3, true>, kMostThreads>(); break;
    case 8:
        if constexpr (LIMIT >= 4) f.template run<SlotWalk<T, 4, false>, kMostThreads>();
        break;
    default:
        if constexpr (LIMIT >= 4) f.template run<SlotWalk<T, 4, true>, kMostThreads>();
        break;
    }
    return true;
}

} // namespace tt
