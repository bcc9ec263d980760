// The residual's addition with a root-mean-square norm behind it (tt_norm_forward), and the gradients (tt_norm_backward).
//
// Both are bound by memory: a value is read once and its results are written once.  A row lies in the registers of a group of lanes
// or of a workgroup, which walks over rows; the next row's vectors are asked for before the present row's sums are joined.
#include <cstdint>
#include "launch_util.h"
#include "norm_math.h"
#include "philox.h"
#include "row_reduce.h"

namespace tt {
namespace {

struct NormParams {
    BlockTable X, R, H, Y; // (R, H: p[0] NULL where there is none)
    const void *gain;
    RowShape r;
    DropParams d;
    float eps;
    uint32_t rows, lanes, groups;
};

// the sum as it is kept: R + dropout(X) in the tensors' type
template <typename T> __device__ __forceinline__ u32x4 sum_of(u32x4 x, u32x4 r, bool res, const DropState &d, uint32_t row, uint32_t col)
{
    constexpr uint32_t EV = kVec<T>;
    if (!res && d.below == 0) return x;
    float f[EV], g[EV];
    unpack16(x, f, T());
    if (d.below) drop_values(d, row, col, f);
    if (res) {
        unpack16(r, g, T());
#pragma unroll
        for (uint32_t e = 0; e < EV; ++e) f[e] += g[e];
    }
    return pack16(f, T());
}

template <typename T, int V, bool WAVE, int MODE>
__global__ __launch_bounds__(WAVE ? kWaveBlock : kMostThreads) void norm_forward_kernel(const NormParams p)
{
    constexpr uint32_t EV = kVec<T>;
    constexpr bool CUT = MODE != kPlain, NARROW = MODE == kNarrow;
    constexpr bool AHEAD = V <= 2, KEPT = V <= 2; // more vectors than that: nothing is asked for ahead, places and gains are worked out and read again
    __shared__ RowScratch<1> scratch;
    const DropState d = drop_state(p.d);
    const uint32_t li = WAVE ? threadIdx.x & (p.lanes - 1) : threadIdx.x;
    const uint32_t at_once = WAVE ? kWaveBlock / p.lanes : 1, step = p.groups * at_once;
    const bool res = p.R.p[0] != nullptr, keep = p.H.p[0] != nullptr;
    Spot spots[KEPT ? V : 1];
    u32x4 gains[KEPT ? V : 1], x[V], r[V];
    auto spot = [&](int i) {
        if constexpr (KEPT) return spots[i];
        uint32_t j = li + i * p.lanes;
        wave::forget(j);
        return spot_of<EV>(p.r, j);
    };
    auto gain_of = [&](int i) {
        if constexpr (KEPT) return gains[i];
        return p.gain ? gain_at<T, MODE>(p.gain, p.r, spot(i)) : ones<T>();
    };
    if constexpr (KEPT) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            spots[i] = spot_of<EV>(p.r, li + i * p.lanes);
            gains[i] = p.gain ? gain_at<T, MODE>(p.gain, p.r, spots[i]) : ones<T>();
        }
    }
    auto row_of = [&](uint32_t base) { return WAVE ? base + threadIdx.x / p.lanes : base; };
    auto load = [&](uint32_t base) { // (a row past the end is the last one again)
        const uint32_t row = row_of(base) < p.rows ? row_of(base) : p.rows - 1;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Spot v = spot(i);
            const Lane l = lane_of<CUT>(p.X, p.r.s, p.r.s.a_shift, row, v);
            x[i] = load_spot<T, NARROW>(p.X, l, v);
            if (res) r[i] = load_spot<T, NARROW>(p.R, l, v);
        }
    };
    uint32_t turn = 0;
    uint32_t base = blockIdx.x * at_once;
    if constexpr (AHEAD) load(base);
    for (; base < p.rows; base += step) {
        const bool live = row_of(base) < p.rows;
        const uint32_t row = live ? row_of(base) : p.rows - 1;
        if constexpr (!AHEAD) load(base);
        u32x4 h[V];
        float sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Spot v = spot(i);
            h[i] = sum_of<T>(x[i], r[i], res, d, row, v.q * p.r.s.seg + v.at);
            if (v.n == 0) h[i] = u32x4{0, 0, 0, 0};
            float f[EV];
            unpack16(h[i], f, T());
#pragma unroll
            for (uint32_t e = 0; e < EV; ++e) sum[0] += v.dup > e ? 0.0f : f[e] * f[e];
            wave::forget(h[i]);
        }
        if constexpr (AHEAD) load(base + step < p.rows ? base + step : base);
        RowReduce<WAVE, float, Sum>::run(sum, p.lanes, scratch, turn++);
        float mean = scaled_mean(sum[0], p.r.cols, p.eps, 1.0f), factor = 1.0f;
        const bool fits = fits_fp32(mean);
        if (WAVE ? wave::ballot(!fits) != 0 : !fits) {
            const float by = factor_for(mean);
            sum[0] = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                wave::forget(h[i]); // (unpacked again: the values are not kept in 32 bits over the sum)
                const Spot v = spot(i);
                float f[EV];
                unpack16(h[i], f, T());
#pragma unroll
                for (uint32_t e = 0; e < EV; ++e) sum[0] += v.dup > e ? 0.0f : f[e] * by * (f[e] * by);
            }
            RowReduce<WAVE, float, Sum>::run(sum, p.lanes, scratch, turn++);
            if (!fits) {
                factor = by;
                mean = scaled_mean(sum[0], p.r.cols, p.eps, by);
            }
        }
        const float root = inverse_root(mean);
        const uint32_t keep_n = live ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            Spot v = spot(i);
            v.n &= keep_n;
            float f[EV], g[EV];
            unpack16(h[i], f, T());
            unpack16(gain_of(i), g, T());
#pragma unroll
            for (uint32_t e = 0; e < EV; ++e) f[e] = f[e] * factor * root * g[e];
            if (keep) store_spot<T, CUT, NARROW>(p.H, lane_of<CUT>(p.H, p.r.s, p.r.s.a_shift, row, v), v, h[i]);
            store_spot<T, CUT, NARROW>(p.Y, lane_of<CUT>(p.Y, p.r.s, p.r.s.b_shift, row, v), v, pack16(f, T()));
        }
    }
}

// Rows that registers do not hold: read once for the sum and once for the results, sums in 64 bits.
template <typename T, bool CUT> __global__ __launch_bounds__(kMostThreads) void norm_forward_long_kernel(const NormParams p)
{
    constexpr uint32_t EV = kVec<T>;
    __shared__ RowScratch<1> scratch;
    const DropState d = drop_state(p.d);
    const bool res = p.R.p[0] != nullptr, keep = p.H.p[0] != nullptr;
    uint32_t turn = 0;
    for (uint32_t row = blockIdx.x; row < p.rows; row += p.groups) {
        double s[1] = {0.0}, root = 0.0;
        for (int pass = 0; pass < 2; ++pass) {
            for (uint32_t j = threadIdx.x; j < p.r.units; j += kMostThreads) {
                const Spot v = spot_of<EV>(p.r, j);
                const Lane l = lane_of<CUT>(p.X, p.r.s, p.r.s.a_shift, row, v);
                const u32x4 x = load_spot<T, false>(p.X, l, v), r = res ? load_spot<T, false>(p.R, l, v) : x;
                const u32x4 h = sum_of<T>(x, r, res, d, row, v.q * p.r.s.seg + v.at);
                float f[EV], g[EV];
                unpack16(h, f, T());
                if (pass == 0) {
#pragma unroll
                    for (uint32_t e = 0; e < EV; ++e) s[0] += v.dup > e ? 0.0 : (double)f[e] * f[e];
                } else {
                    unpack16(p.gain ? gain_at<T, kCut>(p.gain, p.r, v) : ones<T>(), g, T());
#pragma unroll
                    for (uint32_t e = 0; e < EV; ++e) f[e] = (float)(f[e] * root * g[e]);
                    if (keep) store_spot<T, CUT, false>(p.H, l, v, h);
                    store_spot<T, CUT, false>(p.Y, lane_of<CUT>(p.Y, p.r.s, p.r.s.b_shift, row, v), v, pack16(f, T()));
                }
            }
            if (pass == 0) {
                RowReduce<false, double, Sum>::run(s, kMostThreads, scratch, turn++);
                root = inverse_root_wide(s[0] / p.r.cols + p.eps);
            }
        }
    }
}

// workgroups of a launch whose workgroups walk over rows: what the CUs hold at a time
uint32_t groups_of(const RowLaunch &w, int64_t rows)
{
    const int64_t all = (rows + w.at_once - 1) / w.at_once, held = (int64_t)kCUs * (2048 / w.block);
    return (uint32_t)(all < held ? all : held);
}

template <typename T, int MODE> void launch_forward_as(const NormParams &p, const RowLaunch &w, hipStream_t s)
{
    const dim3 grid(p.groups), block(w.block);
    if (w.wave) hipLaunchKernelGGL((norm_forward_kernel<T, 1, true, MODE>), grid, block, 0, s, p);
    else if constexpr (MODE != kNarrow) { // (rows of narrow segments have at most 64 vectors)
        if (w.vectors == 1) hipLaunchKernelGGL((norm_forward_kernel<T, 1, false, MODE>), grid, block, 0, s, p);
        else if (w.vectors == 2) hipLaunchKernelGGL((norm_forward_kernel<T, 2, false, MODE>), grid, block, 0, s, p);
        else if (w.vectors == 4) hipLaunchKernelGGL((norm_forward_kernel<T, 4, false, MODE>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((norm_forward_long_kernel<T, MODE != kPlain>), grid, block, 0, s, p);
    }
}
template <typename T> void launch_forward(const NormParams &p, const RowLaunch &w, hipStream_t s)
{
    if (narrow_segments(p.r, kVec<T>)) launch_forward_as<T, kNarrow>(p, w, s);
    else if (uncut(p.X) && uncut(p.Y)) launch_forward_as<T, kPlain>(p, w, s);
    else launch_forward_as<T, kCut>(p, w, s);
}

// ---------------------------------------------------------------- gradients

struct GradParams {
    BlockTable H, dY, dH, dS, dX; // (dH, dS, dX: p[0] NULL where there is none)
    const void *gain;
    float *parts;                 // a row of sums by column for each wave (WAVE) or workgroup, or NULL
    double *stats;                // (long rows) 1 / root and c of each row
    RowShape r;
    DropParams d;
    float eps;
    uint32_t rows, lanes, groups;
};

// Sums by column over the rows that a group of lanes walks over stay in registers, and leave as one row of partial sums in the end;
// norm_gain_kernel adds these up, in an order that the launch's shape alone sets.
template <typename T, int V, bool WAVE, int MODE>
__global__ __launch_bounds__(WAVE ? kWaveBlock : kMostThreads) void norm_backward_kernel(const GradParams p)
{
    constexpr uint32_t EV = kVec<T>;
    constexpr bool CUT = MODE != kPlain, NARROW = MODE == kNarrow;
    constexpr bool AHEAD = V == 1, KEPT = V == 1;
    __shared__ RowScratch<2> scratch;
    const DropState d = drop_state(p.d);
    const uint32_t li = WAVE ? threadIdx.x & (p.lanes - 1) : threadIdx.x;
    const uint32_t at_once = WAVE ? kWaveBlock / p.lanes : 1, step = p.groups * at_once;
    const bool later = p.dH.p[0] != nullptr, sums = p.dS.p[0] != nullptr, branch = p.dX.p[0] != nullptr;
    Spot spots[KEPT ? V : 1];
    u32x4 gains[KEPT ? V : 1], h[V], y[V], g[V];
    float by_col[V][EV];
    auto spot = [&](int i) {
        if constexpr (KEPT) return spots[i];
        uint32_t j = li + i * p.lanes;
        wave::forget(j);
        return spot_of<EV>(p.r, j);
    };
    auto gain_of = [&](int i) {
        if constexpr (KEPT) return gains[i];
        return p.gain ? gain_at<T, MODE>(p.gain, p.r, spot(i)) : ones<T>();
    };
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (KEPT) {
            spots[i] = spot_of<EV>(p.r, li + i * p.lanes);
            gains[i] = p.gain ? gain_at<T, MODE>(p.gain, p.r, spots[i]) : ones<T>();
        }
#pragma unroll
        for (uint32_t e = 0; e < EV; ++e) by_col[i][e] = 0.0f;
    }
    auto row_of = [&](uint32_t base) { return WAVE ? base + threadIdx.x / p.lanes : base; };
    auto load = [&](uint32_t base) {
        const uint32_t row = row_of(base) < p.rows ? row_of(base) : p.rows - 1;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Spot v = spot(i);
            const Lane l = lane_of<CUT>(p.H, p.r.s, p.r.s.a_shift, row, v);
            h[i] = load_spot<T, NARROW>(p.H, l, v);
            y[i] = load_spot<T, NARROW>(p.dY, lane_of<CUT>(p.dY, p.r.s, p.r.s.b_shift, row, v), v);
            if (later) g[i] = load_spot<T, NARROW>(p.dH, l, v);
        }
    };
    uint32_t turn = 0;
    uint32_t base = blockIdx.x * at_once;
    if constexpr (AHEAD) load(base < p.rows ? base : 0);
    for (; base < p.rows; base += step) {
        const bool live = row_of(base) < p.rows;
        const uint32_t row = live ? row_of(base) : p.rows - 1;
        if constexpr (!AHEAD) load(base);
        u32x4 hc[V], yc[V], gc[V];
        float sum[2] = {0.0f, 0.0f}; // of squares, and of gain dY H
        auto add = [&](int i, float by) {
            const Spot v = spot(i);
            float f[EV], dy[EV], gn[EV];
            unpack16(hc[i], f, T());
            unpack16(yc[i], dy, T());
            unpack16(gain_of(i), gn, T());
#pragma unroll
            for (uint32_t e = 0; e < EV; ++e) {
                const float x = v.dup > e ? 0.0f : f[e] * by;
                sum[0] += x * x;
                sum[1] += v.dup > e ? 0.0f : gn[e] * dy[e] * x;
            }
        };
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool none = spot(i).n == 0 || !live;
            hc[i] = none ? u32x4{0, 0, 0, 0} : h[i];
            yc[i] = none ? u32x4{0, 0, 0, 0} : y[i];
            if (later) gc[i] = g[i];
            add(i, 1.0f);
            wave::forget(hc[i]);
            wave::forget(yc[i]);
        }
        if constexpr (AHEAD) load(base + step < p.rows ? base + step : base);
        RowReduce<WAVE, float, Sum, Sum>::run(sum, p.lanes, scratch, turn++);
        float mean = scaled_mean(sum[0], p.r.cols, p.eps, 1.0f), factor = 1.0f, dot = sum[1];
        const bool fits = fits_fp32(mean);
        if (WAVE ? wave::ballot(!fits) != 0 : !fits) {
            const float by = factor_for(mean);
            sum[0] = sum[1] = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                add(i, by);
                wave::forget(hc[i]);
                wave::forget(yc[i]);
            }
            RowReduce<WAVE, float, Sum, Sum>::run(sum, p.lanes, scratch, turn++);
            if (!fits) {
                factor = by;
                mean = scaled_mean(sum[0], p.r.cols, p.eps, by);
                dot = sum[1];
            }
        }
        const float root = inverse_root(mean), c = root * dot / (float)p.r.cols;
        const uint32_t keep_n = live ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            Spot v = spot(i);
            v.n &= keep_n;
            float f[EV], dy[EV], gn[EV], at[EV];
            unpack16(hc[i], f, T());
            unpack16(yc[i], dy, T());
            unpack16(gain_of(i), gn, T());
            if (later) unpack16(gc[i], at, T());
#pragma unroll
            for (uint32_t e = 0; e < EV; ++e) {
                const float n = f[e] * factor * root;
                if (live) by_col[i][e] += dy[e] * n;
                const float ds = (gn[e] * dy[e] - c * n) * root * factor;
                f[e] = later ? ds + at[e] : ds;
            }
            const Lane l = lane_of<CUT>(p.H, p.r.s, p.r.s.a_shift, row, v);
            if (sums) store_spot<T, CUT, NARROW>(p.dS, l, v, pack16(f, T()));
            if (branch) {
                drop_values(d, row, v.q * p.r.s.seg + v.at, f);
                store_spot<T, CUT, NARROW>(p.dX, l, v, pack16(f, T()));
            }
        }
    }
    if (!p.parts) return;
    // groups of a wave that hold the same columns are joined first
    if constexpr (WAVE) {
        for (uint32_t m = p.lanes; m < 64; m <<= 1) {
#pragma unroll
            for (uint32_t e = 0; e < EV; ++e) by_col[0][e] += lane_xor(by_col[0][e], m);
        }
        if ((threadIdx.x & 63) >= p.lanes) return;
    }
    float *to = p.parts + (size_t)(WAVE ? blockIdx.x * (kWaveBlock / 64) + (threadIdx.x >> 6) : blockIdx.x) * p.r.cols;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const Spot v = spot(i);
#pragma unroll
        for (uint32_t e = 0; e < EV; ++e)
            if (e >= v.dup && e < v.n) store1(to + v.q * p.r.s.seg + v.at + e, by_col[i][e]);
    }
}

// dgain from `count` rows of partial sums: 64 columns a workgroup, a wave takes every 16th row
__global__ __launch_bounds__(kMostThreads) void norm_gain_kernel(const float *parts, uint32_t count, uint32_t cols, float *dgain)
{
    __shared__ float of_wave[kMostWaves][64];
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (uint32_t i = wave; i < count; i += kMostWaves) s += load1(parts + (size_t)i * cols + col);
    }
    of_wave[wave][lane] = s;
    __syncthreads();
    if (wave || col >= cols) return;
    for (int w = 1; w < kMostWaves; ++w) s += of_wave[w][lane];
    store1(dgain + col, s);
}

constexpr uint32_t kLongGroups = 2 * kCUs;

// Rows that registers do not hold: their sums first, then strips of columns, all in 64 bits.
template <typename T, bool CUT> __global__ __launch_bounds__(kMostThreads) void norm_stats_long_kernel(const GradParams p)
{
    constexpr uint32_t EV = kVec<T>;
    __shared__ RowScratch<2> scratch;
    uint32_t turn = 0;
    for (uint32_t row = blockIdx.x; row < p.rows; row += kLongGroups) {
        double s[2] = {0.0, 0.0};
        for (uint32_t j = threadIdx.x; j < p.r.units; j += kMostThreads) {
            const Spot v = spot_of<EV>(p.r, j);
            float f[EV], dy[EV], gn[EV];
            unpack16(load_spot<T, false>(p.H, lane_of<CUT>(p.H, p.r.s, p.r.s.a_shift, row, v), v), f, T());
            unpack16(load_spot<T, false>(p.dY, lane_of<CUT>(p.dY, p.r.s, p.r.s.b_shift, row, v), v), dy, T());
            unpack16(p.gain ? gain_at<T, kCut>(p.gain, p.r, v) : ones<T>(), gn, T());
#pragma unroll
            for (uint32_t e = 0; e < EV; ++e) {
                s[0] += v.dup > e ? 0.0 : (double)f[e] * f[e];
                s[1] += v.dup > e ? 0.0 : (double)gn[e] * dy[e] * f[e];
            }
        }
        RowReduce<false, double, Sum, Sum>::run(s, kMostThreads, scratch, turn++);
        if (threadIdx.x == 0) {
            const double root = inverse_root_wide(s[0] / p.r.cols + p.eps);
            p.stats[2 * (size_t)row] = root;
            p.stats[2 * (size_t)row + 1] = root * s[1] / p.r.cols;
        }
    }
}
template <typename T, bool CUT> __global__ __launch_bounds__(kWaveBlock) void norm_backward_long_kernel(const GradParams p)
{
    constexpr uint32_t EV = kVec<T>;
    const DropState d = drop_state(p.d);
    const bool later = p.dH.p[0] != nullptr, sums = p.dS.p[0] != nullptr, branch = p.dX.p[0] != nullptr;
    const Spot v = spot_of<EV>(p.r, blockIdx.x * kWaveBlock + threadIdx.x);
    if (v.n == 0) return;
    float gn[EV];
    double by_col[EV];
    unpack16(p.gain ? gain_at<T, kCut>(p.gain, p.r, v) : ones<T>(), gn, T());
#pragma unroll
    for (uint32_t e = 0; e < EV; ++e) by_col[e] = 0.0;
    for (uint32_t row = blockIdx.y; row < p.rows; row += p.groups) {
        const double root = load1(p.stats + 2 * (size_t)row), c = load1(p.stats + 2 * (size_t)row + 1);
        const Lane l = lane_of<CUT>(p.H, p.r.s, p.r.s.a_shift, row, v);
        float f[EV], dy[EV], at[EV];
        unpack16(load_spot<T, false>(p.H, l, v), f, T());
        unpack16(load_spot<T, false>(p.dY, lane_of<CUT>(p.dY, p.r.s, p.r.s.b_shift, row, v), v), dy, T());
        if (later) unpack16(load_spot<T, false>(p.dH, l, v), at, T());
#pragma unroll
        for (uint32_t e = 0; e < EV; ++e) {
            const double n = f[e] * root;
            by_col[e] += dy[e] * n;
            f[e] = (float)(((double)gn[e] * dy[e] - c * n) * root + (later ? at[e] : 0.0f));
        }
        if (sums) store_spot<T, CUT, false>(p.dS, l, v, pack16(f, T()));
        if (branch) {
            drop_values(d, row, v.q * p.r.s.seg + v.at, f);
            store_spot<T, CUT, false>(p.dX, l, v, pack16(f, T()));
        }
    }
    if (!p.parts) return;
    float *to = p.parts + (size_t)blockIdx.y * p.r.cols + v.q * p.r.s.seg + v.at;
#pragma unroll
    for (uint32_t e = 0; e < EV; ++e)
        if (e >= v.dup) store1(to + e, (float)by_col[e]);
}

// What a backward launch of so many rows takes: workgroups, and rows of partial sums
struct GradLaunch {
    RowLaunch w;
    uint32_t groups, parts;
    size_t stats_bytes, bytes;
};
// Eight rows a group of lanes where there are many: partial sums are a thirty-second of what is read and written then, and less.
GradLaunch grad_launch(const RowShape &r, int64_t rows)
{
    GradLaunch g;
    g.w = row_launch(r);
    g.stats_bytes = 0;
    if (g.w.vectors == 0) {
        g.groups = (uint32_t)(rows < 64 ? rows : 64); // (of each strip)
        g.parts = g.groups;
        g.stats_bytes = align_up((size_t)rows * 2 * sizeof(double), 256);
    } else {
        const int64_t most = (int64_t)kCUs * (2048 / g.w.block), walks = (rows + g.w.at_once - 1) / g.w.at_once;
        int64_t n = walks / 8;
        if (n < kCUs) n = kCUs;
        if (n > walks) n = walks;
        if (n > most) n = most;
        g.groups = (uint32_t)n;
        g.parts = g.groups * (g.w.wave ? kWaveBlock / 64 : 1);
    }
    g.bytes = rows == 0 || r.cols == 0 ? 0 : g.stats_bytes + align_up((size_t)g.parts * r.cols * sizeof(float), 256);
    return g;
}

template <typename T, int MODE> void launch_backward_as(const GradParams &p, const GradLaunch &g, hipStream_t s)
{
    const dim3 grid(p.groups), block(g.w.block);
    if (g.w.wave) hipLaunchKernelGGL((norm_backward_kernel<T, 1, true, MODE>), grid, block, 0, s, p);
    else if constexpr (MODE != kNarrow) {
        if (g.w.vectors == 1) hipLaunchKernelGGL((norm_backward_kernel<T, 1, false, MODE>), grid, block, 0, s, p);
        else if (g.w.vectors == 2) hipLaunchKernelGGL((norm_backward_kernel<T, 2, false, MODE>), grid, block, 0, s, p);
        else if (g.w.vectors == 4) hipLaunchKernelGGL((norm_backward_kernel<T, 4, false, MODE>), grid, block, 0, s, p);
        else {
            const dim3 rows(p.rows < kLongGroups ? p.rows : kLongGroups), strips((p.r.units + kWaveBlock - 1) / kWaveBlock, g.groups), lanes(kWaveBlock);
            hipLaunchKernelGGL((norm_stats_long_kernel<T, MODE != kPlain>), rows, block, 0, s, p);
            hipLaunchKernelGGL((norm_backward_long_kernel<T, MODE != kPlain>), strips, lanes, 0, s, p);
        }
    }
}
template <typename T> void launch_backward(const GradParams &p, const GradLaunch &g, hipStream_t s)
{
    if (narrow_segments(p.r, kVec<T>)) launch_backward_as<T, kNarrow>(p, g, s);
    else if (uncut(p.H) && uncut(p.dY)) launch_backward_as<T, kPlain>(p, g, s);
    else launch_backward_as<T, kCut>(p, g, s);
}

// the geometry of a backward call (shard lists may be NULL)
tt_status grad_shape(int64_t rows, int64_t width, int k, int dtype, const tt_tiling &tX, const tt_tiling &tdY, const void *const *H, const void *const *dY,
                     GradParams *p)
{
    if (!valid_k(k) || !valid_tiling(tX, k) || !valid_tiling(tdY, k) || !valid_dtype(dtype) || rows < 0 || width < 0) return TT_EINVAL;
    if (!fits31(rows) || !fits31(width)) return TT_EUNSUPPORTED;
    if (!make_blocks(H, tX, k, rows, width, &p->H) || !make_blocks(dY, tdY, k, rows, width, &p->dY)) return TT_EINFEASIBLE;
    p->rows = (uint32_t)rows;
    if (width == 0) p->r = RowShape{};
    else p->r = row_shape(p->H, p->dY, width, 16 / dtype_bytes(dtype));
    return TT_OK;
}

bool valid_eps(float eps) { return eps > 0.0f && eps <= 3.4e38f; }
const void *const *in(void *const *p) { return const_cast<const void *const *>(p); }

} // namespace
} // namespace tt

extern "C" tt_status tt_norm_forward(int64_t rows, int64_t width, int k, int dtype, tt_tiling tX, tt_tiling tY, float eps, const tt_drop *drop,
                                     const void *const *X, const void *const *R, const void *gain, void *const *H, void *const *Y, void *stream)
{
    using namespace tt;
    NormParams p;
    if (!make_drop(drop, &p.d) || !valid_eps(eps)) return TT_EINVAL;
    if (!valid_k(k) || !valid_tiling(tX, k) || !valid_tiling(tY, k) || !valid_dtype(dtype) || rows < 0 || width < 0) return TT_EINVAL;
    const bool empty = rows == 0 || width == 0;
    const int e = dtype_bytes(dtype);
    if (!shards_fit(X, k, e, empty) || (R && !shards_fit(R, k, e, empty)) || (H && !shards_fit(in(H), k, e, empty)) || !shards_fit(in(Y), k, e, empty))
        return TT_EINVAL;
    if (gain && !aligned_to(gain, e)) return TT_EINVAL;
    if (!fits31(rows) || !fits31(width)) return TT_EUNSUPPORTED;
    if (!make_blocks(X, tX, k, rows, width, &p.X) || !make_blocks(R, tX, k, rows, width, &p.R) || !make_blocks(in(H), tX, k, rows, width, &p.H) ||
        !make_blocks(in(Y), tY, k, rows, width, &p.Y))
        return TT_EINFEASIBLE;
    if (empty) return TT_OK;
    p.gain = gain;
    p.eps = eps;
    p.rows = (uint32_t)rows;
    p.r = row_shape(p.X, p.Y, width, 16 / e);
    const RowLaunch w = row_launch(p.r);
    p.lanes = w.lanes;
    p.groups = groups_of(w, rows);
    ProfileScope scope(stream, TT_K_NORM, 1 << k, rows, width, e, (uint64_t)rows * width * e * (1 + (R ? 1 : 0) + (H ? p.H.nrep : 0) + p.Y.nrep), 0);
    if (dtype == TT_BF16) launch_forward<uint16_t>(p, w, static_cast<hipStream_t>(stream));
    else launch_forward<float>(p, w, static_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
}

extern "C" tt_status tt_norm_workspace_bytes(int64_t rows, int64_t width, int k, int dtype, tt_tiling tX, tt_tiling tdY, size_t *bytes)
{
    using namespace tt;
    GradParams p;
    if (!bytes) return TT_EINVAL;
    const tt_status st = grad_shape(rows, width, k, dtype, tX, tdY, nullptr, nullptr, &p);
    if (st != TT_OK) return st;
    *bytes = rows == 0 || width == 0 ? 0 : grad_launch(p.r, rows).bytes;
    return TT_OK;
}

extern "C" tt_status tt_norm_backward(int64_t rows, int64_t width, int k, int dtype, tt_tiling tX, tt_tiling tdY, float eps, const tt_drop *drop,
                                      const void *const *H, const void *gain, const void *const *dY, const void *const *dH, void *const *dS,
                                      void *const *dX, float *dgain, void *workspace, size_t ws_bytes, void *stream)
{
    using namespace tt;
    GradParams p;
    if (!make_drop(drop, &p.d) || !valid_eps(eps) || (dX && !drop)) return TT_EINVAL;
    const tt_status st = grad_shape(rows, width, k, dtype, tX, tdY, H, dY, &p);
    if (st != TT_OK && st != TT_EINFEASIBLE) return st;
    const bool empty = rows == 0 || width == 0;
    const int e = dtype_bytes(dtype);
    if (!shards_fit(H, k, e, empty) || !shards_fit(dY, k, e, empty) || (dH && !shards_fit(dH, k, e, empty)) ||
        (dS && !shards_fit(in(dS), k, e, empty)) || (dX && !shards_fit(in(dX), k, e, empty)))
        return TT_EINVAL;
    if ((gain && !aligned_to(gain, e)) || (dgain && !aligned_to(dgain, 4))) return TT_EINVAL;
    if (st != TT_OK) return st;
    make_blocks(dH, tX, k, rows, width, &p.dH);
    make_blocks(in(dS), tX, k, rows, width, &p.dS);
    make_blocks(in(dX), tX, k, rows, width, &p.dX);
    if (width == 0) return TT_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 strips((uint32_t)((width + 63) / 64)), threads(kMostThreads);
    if (empty) { // a gradient of zeros: the sum of no rows
        if (!dgain) return TT_OK;
        hipLaunchKernelGGL(norm_gain_kernel, strips, threads, 0, s, static_cast<const float *>(nullptr), 0u, (uint32_t)width, dgain);
        return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
    }
    const GradLaunch g = grad_launch(p.r, rows);
    if (!workspace || ws_bytes < g.bytes || reinterpret_cast<uintptr_t>(workspace) % 256) return TT_EWORKSPACE;
    if (!dS && !dX && !dgain) return TT_OK;
    p.gain = gain;
    p.eps = eps;
    p.lanes = g.w.lanes;
    p.groups = g.groups;
    p.stats = static_cast<double *>(workspace);
    float *parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + g.stats_bytes);
    p.parts = dgain ? parts : nullptr;
    const uint64_t values = (uint64_t)rows * width * e;
    {
        ProfileScope scope(stream, TT_K_NORM_GRAD, 1 << k, rows, width, e, values * (2 + (dH ? 1 : 0) + ((dS ? 1 : 0) + (dX ? 1 : 0)) * p.H.nrep), 0);
        if (dtype == TT_BF16) launch_backward<uint16_t>(p, g, s);
        else launch_backward<float>(p, g, s);
    }
    if (dgain) {
        ProfileScope scope(stream, TT_K_NORM_GRAD, 1, g.parts, width, 4, (uint64_t)g.parts * width * 4, 0);
        hipLaunchKernelGGL(norm_gain_kernel, strips, threads, 0, s, const_cast<const float *>(parts), g.parts, (uint32_t)width, dgain);
    }
    return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
}
