// The clipped policy loss on a chain's logits and its gradient, and the tokens' log probabilities alone.
//
// A row of logits gives one number, log p[a] = z_a - log sum exp z, and with its derivative g of the loss the row's gradient
// g (onehot(a) - p): two sums over the row and a pass that writes as much as was read.  Memory bounds it (8 flops and two
// exponentials a value), so the logits are to come from memory once: 4096 x 131072 bf16 logits, 1.075 GB read and 1.074 written in
// 418 us, 5.1 TB/s.  Log probabilities alone: 4096 x 131072 177 us, 6.1 TB/s; 16 x 131072 8.2 us on the GPU, trips to memory.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>
#include "launch_util.h"
#include "tiled_rows.h"

namespace tt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Statistics of a part of a row, in base 2: the sum of 2^((x - top) kk) over it, top its largest logit as it is stored.  The
// difference comes first: near the maximum it is exact and for the maximum itself 0, however large the logits are (the rounding
// of a product x kk would be worth more than a power of 2 from some 1e9 on, and the product infinite for a mask of the type's lowest
// value).  A part with nothing above -inf has top -inf and a sum of 0, or NaN where it holds one.
struct Stats { float top, sum; };
__device__ __forceinline__ float power_of(float x, float top, float kk) { return wave::exp2_fast((x - top) * kk); }

struct PolicyParams {
    BlockTable X, G;
    Pieces s;
    Divisor by_ups;        // units (64 neighbouring vectors, one a lane of a wave) that are whole in a segment,
    uint32_t units;        // ... in a row
    uint32_t rest;         // vectors of a segment behind its whole units
    const void *actions;
    uint32_t wide_ids, with_dx;
    const float *old_logp, *ref_logp, *advantage, *weight; // weight NULL: log probabilities alone
    float *logp, *row_loss;                                // either may be NULL
    float *loss;                                           // NULL: log probabilities alone
    Stats *part_stats;                                     // [tokens][parts], where rows are cut
    uint32_t parts;
    Divisor by_parts;
    uint32_t tokens, groups; // rows, and the workgroups that share them
    int64_t vocab;
    tt_policy policy;
};

__device__ __forceinline__ int64_t action_of(const PolicyParams &p, uint32_t t)
{
    return p.wide_ids ? token_scalar<int64_t>(p.actions, t) : token_scalar<int32_t>(p.actions, t);
}
// whether a token counts as far as its weight and action go
__device__ __forceinline__ bool counts(const PolicyParams &p, uint32_t t, int64_t a) { return a >= 0 && a < p.vocab && !(p.weight && load_scalar(p.weight + t) == 0.0f); }

// power_of with what rounding the product leaves out put right, where statistics are joined: bf16 logits lie at few distances from
// each other, so that the same roundings would come in every row.
__device__ __forceinline__ float join_power(float x, float top, float kk)
{
    const float d = x - top, e = d * kk;
    return e > -150.0f ? wave::exp2_fast(e) * fmaf(fmaf(d, kk, -e), 0.693147181f, 1.0f) : 0.0f;
}
// log2(e) times the logits' factor (finite, so that it is no power at all for the maximum)
__device__ __forceinline__ float exponent_factor(const PolicyParams &p) { return fminf(p.policy.scale * kLog2e, 3.402823466e38f); }

__device__ __forceinline__ Stats joined(Stats a, Stats b, float kk)
{
    const float top = fmaxf(a.top, b.top);
    const float fa = a.top == -INFINITY ? 1.0f : join_power(a.top, top, kk), fb = b.top == -INFINITY ? 1.0f : join_power(b.top, top, kk);
    return {top, a.sum * fa + b.sum * fb};
}
__device__ __forceinline__ Stats wave_joined(Stats s, float kk)
{
    const float top = wave_max(s.top);
    return {top, wave_sum(s.top == -INFINITY ? s.sum : s.sum * join_power(s.top, top, kk))};
}
// over a workgroup's waves, in every thread; `red`: a Stats per wave
template <int WAVES> __device__ __forceinline__ Stats group_joined(Stats s, Stats *red, float kk)
{
    s = wave_joined(s, kk);
    if ((threadIdx.x & 63u) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    return wave_joined((threadIdx.x & 63u) < (uint32_t)WAVES ? red[threadIdx.x & 63u] : Stats{-INFINITY, 0.0f}, kk);
}

template <typename T> __device__ __forceinline__ float max_of(u32x4 v, float m)
{
    float f[kVec<T>];
    unpack16(v, f, T());
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) m = fmaxf(m, f[i]);
    return m;
}
// 2^((x - top) kk) for many x: whole() of the sum of of(x).  fp32: power_of.  bf16, where the arithmetic is what a row waits for,
// a fused step in place of two (difference first throughout: 1000 x 50021 47.4 us, so 46.2): of(x) = 2^(x kk - c) with c the rounded
// top kk, whole() puts right what the rounding left out, 2^-7 of an exponent at most.  Beyond |top| kk = 2^18 a smaller factor keeps c
// below it: numbers of 8 bits that are not top are 2^-8 of it away at least, 2^9 as an exponent, and have no power, as by kk itself.
template <typename T> struct Powers {
    float kk, top, c;
    __device__ __forceinline__ Powers(float k, float t) : kk(k), top(t), c(0.0f)
    {
        if constexpr (sizeof(T) == 2) {
            if (fabsf(top) * kk > 262144.0f) kk = __uint_as_float((127u + 17u + 127u - ((__float_as_uint(top) >> 23) & 255u)) << 23);
            c = top * kk;
        }
    }
    // (the exponential's series: a power next to 1 would be rounded to steps as large as what it puts right)
    __device__ __forceinline__ float whole(float s) const
    {
        if (sizeof(T) != 2) return s;
        const float t = fmaf(top, kk, -c) * 0.693147181f;
        return fmaf(s * t, fmaf(t, fmaf(t, -1.0f / 6, 0.5f), -1.0f), s);
    }
    __device__ __forceinline__ float of(float x) const { return sizeof(T) == 2 ? wave::exp2_fast(fmaf(x, kk, -c)) : power_of(x, top, kk); }
};
template <typename T, class F> __device__ __forceinline__ float sum_of(u32x4 v, F &&of, float s)
{
    float f[kVec<T>];
    unpack16(v, f, T());
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) s += of(f[i]);
    return s;
}

// What a row's statistics come to: its log probability, its part of the loss, the factor of p's numerators in its gradient and
// what the action's entry has on top.  A few scalars a row, with log p and its differences from the old and the reference one
// taken in 64 bits: the loss is a sum of terms of both signs.
struct RowResult { float logp, loss, coef, at_a; bool live; };
struct TokenScalars { float weight, old_logp, ref_logp, advantage; };
__device__ __forceinline__ TokenScalars scalars_of(const PolicyParams &p, uint32_t t)
{
    TokenScalars c{0.0f, 0.0f, 0.0f, 0.0f};
    if (!p.weight) return c;
    c.weight = load_scalar(p.weight + t);
    c.old_logp = load_scalar(p.old_logp + t);
    c.advantage = load_scalar(p.advantage + t);
    if (p.policy.kl != 0.0f) c.ref_logp = load_scalar(p.ref_logp + t);
    return c;
}
__device__ __forceinline__ RowResult row_result(const PolicyParams &p, const TokenScalars &c, Stats s, float xa, float kk)
{
    RowResult r{0.0f, 0.0f, 0.0f, 0.0f, true};
    if (s.top == -INFINITY && s.sum == 0.0f) { // nothing above -inf
        r.live = false;
        return r;
    }
    int e = 0;
    const float f = frexpf(s.sum, &e); // log2 of a number next to 1, and a whole number
    // (by kk, as the sum's powers go: the action's logit and the others are off by the same part of 10^-8, which cancels but for how far
    // the action lies from the mean of p)
    const double lp = (((double)xa - (double)s.top) * (double)kk - (double)e - (double)log2f(f)) * 0.6931471805599453;
    r.logp = (float)lp;
    if (!p.weight) return r;
    const float w = c.weight, adv = c.advantage, lo = 1.0f - p.policy.clip_low, hi = 1.0f + p.policy.clip_high;
    const float ratio = expf((float)(lp - (double)c.old_logp));
    const float clipped = ratio < lo ? lo : ratio > hi ? hi : ratio;
    const float a = ratio * adv, b = clipped * adv;
    float loss = a < b || a != a ? -a : -b;
    const bool held = (adv > 0.0f && ratio > hi) || (adv < 0.0f && ratio < lo);
    float d = held ? 0.0f : -a;
    if (p.policy.kl != 0.0f) {
        const float diff = (float)((double)c.ref_logp - lp), em1 = expm1f(diff);
        loss += p.policy.kl * (em1 - diff);
        d -= p.policy.kl * em1;
    }
    r.loss = w * loss;
    r.at_a = w * d * p.policy.scale;
    r.coef = -r.at_a / s.sum;
    return r;
}
__device__ __forceinline__ void store_scalars(const PolicyParams &p, uint32_t t, const RowResult &r)
{
    if (p.logp) p.logp[t] = r.logp;
    if (p.row_loss) p.row_loss[t] = r.loss;
}

// statistics with N more vectors (vectors of -inf add nothing)
template <typename T, int N> __device__ __forceinline__ Stats with_vectors(Stats s, const u32x4 *r, float kk)
{
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max_of<T>(r[i], m);
    const float top = fmaxf(s.top, m), from = top == -INFINITY ? 0.0f : top;
    float sum = s.top == -INFINITY ? s.sum : s.sum * power_of(s.top, from, kk);
    if constexpr (N > 1 && sizeof(T) == 2) { // (for one vector what Powers saves is less than what it takes)
        const Powers<T> e(kk, from);
        float more = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) more = sum_of<T>(r[i], [&](float x) { return e.of(x); }, more);
        return {top, sum + e.whole(more)};
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sum = sum_of<T>(r[i], [&](float x) { return power_of(x, from, kk); }, sum);
    return {top, sum};
}

// coef 2^((x - top) kk) over a row
template <typename T> struct Gradient {
    Powers<T> e;
    float coef;
    __device__ __forceinline__ Gradient(float kk, float top, float c) : e(kk, top), coef(c)
    {
        coef = e.whole(coef);
        e.kk = __uint_as_float(uniform(__float_as_uint(e.kk)));
    }
    __device__ __forceinline__ u32x4 of(u32x4 v) const
    {
        float f[kVec<T>];
        unpack16(v, f, T());
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) f[i] = coef * e.of(f[i]);
        return pack16(f, T());
    }
};

// Where whole unit u of a row lies: segment and first vector
struct Unit { uint32_t q, j0; };
__device__ __forceinline__ Unit unit_of(const PolicyParams &p, uint32_t u)
{
    const uint32_t q = p.s.nseg == 1 ? 0 : quotient(u, p.by_ups);
    return {q, (u - q * p.by_ups.d) * 64};
}
template <typename T> __device__ __forceinline__ u32x4 load_unit(const PolicyParams &p, uint32_t t, uint32_t u)
{
    const Unit g = unit_of(p, u);
    const T *src = source_of<T>(p.X, p.s, p.s.a_shift, t, g.q) + g.j0 * kVec<T>;
    return load16(src + (threadIdx.x & 63u) * kVec<T>);
}
template <typename T> __device__ __forceinline__ void store_unit(const PolicyParams &p, uint32_t t, uint32_t u, u32x4 v)
{
    const Unit g = unit_of(p, u);
    const Place to = place_of(p.G, p.s, p.s.b_shift, t, g.q);
    for (uint32_t x = 0; x < p.G.nrep; ++x) {
        T *dst = static_cast<T *>(p.G.p[to.block + x]) + to.at + g.j0 * kVec<T>;
        store16_once(dst + (threadIdx.x & 63u) * kVec<T>, v);
    }
}

template <typename T> constexpr uint32_t kNothing = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u; // -inf
// The rest of segment q, up to 64 vectors of which the last may be short.  Every lane loads a whole vector: a short one those
// values that end with the segment, what is not its own in front of them; lanes past the end the same.  only_own() then
// puts -inf in the place of what is not a lane's own.  (Segments of less than a vector: any_rest.)
template <typename T> __device__ __forceinline__ uint32_t rest_column(const PolicyParams &p)
{
    const uint32_t c = (p.by_ups.d * 64 + (threadIdx.x & 63u)) * kVec<T>, last = p.s.seg - kVec<T>;
    return c < last ? c : last;
}
template <typename T> __device__ __forceinline__ u32x4 load_rest(const PolicyParams &p, uint32_t t, uint32_t q)
{
    return load16(source_of<T>(p.X, p.s, p.s.a_shift, t, q) + rest_column<T>(p));
}
template <typename T> __device__ __forceinline__ u32x4 only_own(const PolicyParams &p, u32x4 v)
{
    const uint32_t n = values_of(p.s, kVec<T>, p.by_ups.d * 64 + (threadIdx.x & 63u)), skip = kVec<T> - n; // values in front
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            if (2 * i + 1 < (int)skip) v[i] = kNothing<T>;
            else if (2 * i < (int)skip) v[i] = (v[i] & 0xffff0000u) | (kNothing<T> & 0xffffu);
        } else if (i < (int)skip) {
            v[i] = kNothing<T>;
        }
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store_rest(const PolicyParams &p, uint32_t t, uint32_t q, u32x4 v)
{
    const uint32_t n = values_of(p.s, kVec<T>, p.by_ups.d * 64 + (threadIdx.x & 63u));
    if (n == 0) return;
    const Place to = place_of(p.G, p.s, p.s.b_shift, t, q);
    for (uint32_t x = 0; x < p.G.nrep; ++x) {
        T *dst = static_cast<T *>(p.G.p[to.block + x]) + to.at + rest_column<T>(p);
        if (n == (uint32_t)kVec<T>) {
            store16(dst, v);
            continue;
        }
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) {
            if ((uint32_t)i < kVec<T> - n) continue;
            if constexpr (sizeof(T) == 2) store1(dst + i, (uint16_t)(v[i >> 1] >> (16 * (i & 1))));
            else store1(dst + i, __uint_as_float(v[i]));
        }
    }
}
// ... a vector at a time of any segment, its values at the front
template <typename T> __device__ __forceinline__ u32x4 any_rest(const PolicyParams &p, uint32_t t, uint32_t q)
{
    u32x4 r = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
    const uint32_t j = p.by_ups.d * 64 + (threadIdx.x & 63u), n = values_of(p.s, kVec<T>, j);
    if (n == 0) return r;
    const T *src = source_of<T>(p.X, p.s, p.s.a_shift, t, q) + j * kVec<T>;
    if (n == (uint32_t)kVec<T>) return load16(src);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) {
        if ((uint32_t)i >= n) continue;
        if constexpr (sizeof(T) == 2) r[i >> 1] = i & 1 ? (r[i >> 1] & 0xffffu) | (uint32_t)load1(src + i) << 16 : (r[i >> 1] & 0xffff0000u) | load1(src + i);
        else r[i] = __float_as_uint(load1(src + i));
    }
    return r;
}
template <typename T> __device__ __forceinline__ void store_any_rest(const PolicyParams &p, uint32_t t, uint32_t q, u32x4 v)
{
    const uint32_t j = p.by_ups.d * 64 + (threadIdx.x & 63u), n = values_of(p.s, kVec<T>, j);
    if (n) store_all<T>(p.G, place_of(p.G, p.s, p.s.b_shift, t, q), j * kVec<T>, n, v);
}

// where column c of a row lies
struct Column { uint32_t q, offset; };
__device__ __forceinline__ Column column_of(const PolicyParams &p, uint32_t c)
{
    const uint32_t q = p.s.nseg == 1 ? 0 : c / p.s.seg;
    return {q, c - q * p.s.seg};
}
template <typename T> __device__ __forceinline__ T logit_at(const PolicyParams &p, uint32_t t, const Column &c)
{
    return load1(source_of<T>(p.X, p.s, p.s.a_shift, t, c.q) + c.offset);
}
template <typename T> __device__ __forceinline__ void store_entry(const PolicyParams &p, uint32_t t, const Column &c, float v)
{
    const Place to = place_of(p.G, p.s, p.s.b_shift, t, c.q);
    for (uint32_t x = 0; x < p.G.nrep; ++x) store1(static_cast<T *>(p.G.p[to.block + x]) + to.at + c.offset, from_float<T>(v));
}
// The action's entry once more, with what it has on top, by the thread that wrote the vector it lies in: its later store of the two.
template <typename T, int WAVES> __device__ __forceinline__ void store_action(const PolicyParams &p, uint32_t t, const Column &c, float v)
{
    const uint32_t j = c.offset / kVec<T>, unit = j / 64, wave = unit < p.by_ups.d ? (c.q * p.by_ups.d + unit) % WAVES : c.q % WAVES;
    if (threadIdx.x == wave * 64 + (j & 63u)) store_entry<T>(p, t, c, v);
}

// Where the units of a row lie.  Rows that no cut splits: behind the row's first value, worked out once a row.  Otherwise the
// tables of blocks wait in LDS (an address out of the kernel's arguments would be a trip to memory per unit).
template <typename T> struct RowMap {
    const uint64_t *x_table, *g_table;
    __device__ __forceinline__ const T *x_row(const PolicyParams &p, uint32_t t) const { return p.s.nseg == 1 ? source_of<T>(p.X, p.s, p.s.a_shift, t, 0) : nullptr; }
    __device__ __forceinline__ T *g_row(const PolicyParams &p, uint32_t t) const
    {
        if (p.s.nseg > 1 || p.G.nrep > 1) return nullptr;
        const Place to = place_of(p.G, p.s, p.s.b_shift, t, 0);
        return static_cast<T *>(p.G.p[to.block]) + to.at;
    }
    __device__ __forceinline__ u32x4 load(const PolicyParams &p, uint32_t t, const T *row, uint32_t u) const
    {
        const T *src = row + (size_t)u * 64 * kVec<T>;
        if (p.s.nseg > 1) {
            const Unit g = unit_of(p, u);
            const Place at = place_of(p.X, p.s, p.s.a_shift, t, g.q);
            src = reinterpret_cast<const T *>((uintptr_t)uniform(x_table[at.block])) + at.at + g.j0 * kVec<T>;
        }
        return load16(src + (threadIdx.x & 63u) * kVec<T>);
    }
    __device__ __forceinline__ void store(const PolicyParams &p, uint32_t t, T *row, uint32_t u, u32x4 v) const
    {
        const uint32_t lane = threadIdx.x & 63u;
        if (row) {
            store16_once(row + (size_t)u * 64 * kVec<T> + lane * kVec<T>, v);
            return;
        }
        const Unit g = unit_of(p, u);
        const Place to = place_of(p.G, p.s, p.s.b_shift, t, g.q);
        for (uint32_t x = 0; x < p.G.nrep; ++x)
            store16_once(reinterpret_cast<T *>((uintptr_t)uniform(g_table[to.block + x])) + to.at + g.j0 * kVec<T> + lane * kVec<T>, v);
    }
};

// A row in the registers of a workgroup: up to NC vectors a thread of whole units, unit i * WAVES + w with wave w, and the rest of
// segment w with it as well.  The row is read once, for its statistics and for its gradient.  Workgroups stay and take every
// groups-th row: as a vector's gradient leaves, the next row's vector is fetched into its registers, so that memory always
// has work while the workgroup computes.  A row's result (a few hundred instructions, logarithms and exponentials to their last
// bits) is one wave's work.
// Vectors that are taken into the statistics at a time: 4, or 2 beside 20 waiting ones, where 4 would leave 32 registers in memory
// (2048 x 151936 bf16: 267 us, so 259)
constexpr int together_of(int nc) { return nc > 16 ? 2 : nc < 4 ? nc : 4; }
template <typename T, int WAVES, int NC, bool GRAD> __global__ __launch_bounds__(WAVES * 64) void policy_rows_kernel(const PolicyParams p)
{
    __shared__ Stats red[WAVES];
    __shared__ float shared[4]; // top, coef, the action's entry, whether the row counts
    __shared__ uint64_t tables[2][kMaxShards];
    const uint32_t w = uniform(threadIdx.x >> 6);
    const float kk = exponent_factor(p);
    const bool has_rest = p.rest && w < p.s.nseg;
    if (p.s.nseg > 1 || p.G.nrep > 1) {
        if (threadIdx.x < (uint32_t)kMaxShards) {
            tables[0][threadIdx.x] = (uint64_t)(uintptr_t)p.X.p[threadIdx.x];
            tables[1][threadIdx.x] = (uint64_t)(uintptr_t)p.G.p[threadIdx.x];
        }
        __syncthreads();
    }
    const RowMap<T> map{tables[0], tables[1]};
    const u32x4 nothing = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>}, zero = u32x4{0, 0, 0, 0};
    // Slots past the row's units load its last unit again, and nothing is done with them: a load that a branch may skip could not be
    // counted, and every wait would be one for all that is on its way.
    const uint32_t last = p.units - 1;
    const auto slot = [&](int i) {
        uint32_t u = i * WAVES + w;
        u = u < last ? u : last;
        wave::forget_uniform(u); // (addresses are worked out where they are used and not kept for all NC)
        return u;
    };
    uint32_t t = blockIdx.x;
    int64_t a = action_of(p, t);
    bool in = counts(p, t, a);
    TokenScalars c = scalars_of(p, t);
    u32x4 r[NC], rest = nothing;
#pragma unroll
    for (int i = 0; i < NC; ++i) r[i] = nothing;
    if (in) {
        const T *row = map.x_row(p, t);
        if (has_rest) rest = load_rest<T>(p, t, w);
        if (p.units) {
#pragma unroll
            for (int i = 0; i < NC; ++i) r[i] = map.load(p, t, row, slot(i));
        }
    }
    for (;;) {
        const uint32_t next = t + p.groups;
        const bool more = next < p.tokens;
        const int64_t next_a = more ? action_of(p, next) : -1;
        const bool next_in = more && counts(p, next, next_a);
        const TokenScalars next_c = more ? scalars_of(p, next) : TokenScalars{0.0f, 0.0f, 0.0f, 0.0f};
        const T *next_row = next_in ? map.x_row(p, next) : nullptr;
        RowResult res{0.0f, 0.0f, 0.0f, 0.0f, false};
        Column ca{0, 0};
        float top = 0.0f, entry = 0.0f;
        if (in) {
            ca = column_of(p, (uint32_t)a);
            const T xa = logit_at<T>(p, t, ca);
            // in the order in which the vectors were fetched, a few at a time: the later ones are still on their way
            Stats s{-INFINITY, 0.0f};
            if (has_rest) {
                rest = only_own<T>(p, rest);
                s = with_vectors<T, 1>(s, &rest, kk);
            }
#pragma unroll
            for (int i = 0; i < NC; i += together_of(NC)) {
                constexpr int most = together_of(NC);
#pragma unroll
                for (int k = i; k < i + most; ++k)
                    if (k * WAVES + w >= p.units) r[k] = nothing;
                s = with_vectors<T, most>(s, r + i, kk);
                if constexpr (!GRAD) { // nobody needs them again
                    if (next_in && p.units) {
#pragma unroll
                        for (int k = i; k < i + most; ++k) r[k] = map.load(p, next, next_row, slot(k));
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            s = wave_joined(s, kk);
            if constexpr (GRAD) {
#pragma unroll
                for (int i = 0; i < NC; ++i) wave::forget(r[i]);
            }
            if constexpr (WAVES > 1) {
                if ((threadIdx.x & 63u) == 0) red[w] = s;
                __syncthreads();
            }
            if (w == 0) {
                if constexpr (WAVES > 1) {
                    const uint32_t lane = threadIdx.x & 63u;
                    s = wave_joined(lane < (uint32_t)WAVES ? red[lane] : Stats{-INFINITY, 0.0f}, kk);
                }
                const float x = to_float(xa);
                res = row_result(p, c, s, x, kk);
                top = s.top;
                entry = fmaf(res.coef, power_of(x, top, kk), res.at_a);
                if (threadIdx.x == 0) {
                    store_scalars(p, t, res);
                    if constexpr (WAVES > 1 && GRAD) {
                        shared[0] = top;
                        shared[1] = res.coef;
                        shared[2] = entry;
                        shared[3] = res.live ? 1.0f : 0.0f;
                    }
                }
            }
            if constexpr (WAVES > 1) __syncthreads();
            if constexpr (WAVES > 1 && GRAD) {
                top = shared[0];
                res.coef = shared[1];
                entry = shared[2];
                res.live = shared[3] != 0.0f;
            }
        } else if (threadIdx.x == 0) {
            store_scalars(p, t, res);
        }
        if constexpr (GRAD) {
            T *row = map.g_row(p, t);
            const Gradient<T> grad(kk, top, res.coef);
            // Everything fetched so far is here and used; said once, or the compiler, which cannot tell for rows that do not
            // count, waits for every store in front of each of the next row's loads.
            __builtin_amdgcn_s_waitcnt(0x0f70); // vmcnt(0)
            const auto emit = [&](auto fetch) {
                if (has_rest) {
                    const u32x4 g = res.live ? grad.of(rest) : zero;
                    if constexpr (decltype(fetch)::value) rest = load_rest<T>(p, next, w);
                    store_rest<T>(p, t, w, g);
                }
                if (p.units == 0) return;
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const u32x4 g = res.live ? grad.of(r[i]) : zero;
                    if constexpr (decltype(fetch)::value) r[i] = map.load(p, next, next_row, slot(i));
                    if (i * WAVES + w < p.units) map.store(p, t, row, i * WAVES + w, g);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            if (next_in) emit(std::true_type());
            else emit(std::false_type());
            if (res.live) store_action<T, WAVES>(p, t, ca, entry);
        } else if (next_in) {
            if (!in && p.units) {
#pragma unroll
                for (int i = 0; i < NC; ++i) r[i] = map.load(p, next, next_row, slot(i));
            }
            if (has_rest) rest = load_rest<T>(p, next, w);
        }
        if (!more) break;
        t = next;
        a = next_a;
        in = next_in;
        c = next_c;
    }
}

// Rows that do not fit: one workgroup per row, which reads it for its statistics and again for its gradient (from the caches,
// where they hold it).  1024 x 200000 bf16: 196 us, 4.2 TB/s of what has to move; 1000 x 100000 fp32: 193, 4.1.
constexpr int kStreamWaves = 16;
template <typename T> __global__ __launch_bounds__(kStreamWaves * 64) void policy_stream_kernel(const PolicyParams p)
{
    constexpr int U = 4;
    __shared__ Stats red[kStreamWaves];
    const uint32_t t = blockIdx.x, w = uniform(threadIdx.x >> 6);
    const int64_t a = action_of(p, t);
    const float kk = exponent_factor(p);
    RowResult res{0.0f, 0.0f, 0.0f, 0.0f, false};
    Stats s{-INFINITY, 0.0f};
    Column ca{0, 0};
    float xa = 0.0f;
    if (counts(p, t, a)) {
        ca = column_of(p, (uint32_t)a);
        xa = to_float(logit_at<T>(p, t, ca));
        uint32_t u = w;
        for (; u + (U - 1) * kStreamWaves < p.units; u += U * kStreamWaves) {
            u32x4 r[U];
#pragma unroll
            for (int i = 0; i < U; ++i) r[i] = load_unit<T>(p, t, u + i * kStreamWaves);
            s = with_vectors<T, U>(s, r, kk);
        }
        for (; u < p.units; u += kStreamWaves) {
            const u32x4 r = load_unit<T>(p, t, u);
            s = with_vectors<T, 1>(s, &r, kk);
        }
        if (p.rest)
            for (uint32_t q = w; q < p.s.nseg; q += kStreamWaves) {
                const u32x4 r = any_rest<T>(p, t, q);
                s = with_vectors<T, 1>(s, &r, kk);
            }
        s = group_joined<kStreamWaves>(s, red, kk);
        res = row_result(p, scalars_of(p, t), s, xa, kk);
    }
    if (threadIdx.x == 0) store_scalars(p, t, res);
    if (!p.with_dx) return;
    const Gradient<T> grad(kk, s.top, res.coef);
    const u32x4 zero = u32x4{0, 0, 0, 0};
    uint32_t u = w;
    for (; u + (U - 1) * kStreamWaves < p.units; u += U * kStreamWaves) {
        u32x4 r[U];
#pragma unroll
        for (int i = 0; i < U; ++i) r[i] = res.live ? load_unit<T>(p, t, u + i * kStreamWaves) : zero;
#pragma unroll
        for (int i = 0; i < U; ++i) store_unit<T>(p, t, u + i * kStreamWaves, res.live ? grad.of(r[i]) : zero);
    }
    for (; u < p.units; u += kStreamWaves) store_unit<T>(p, t, u, res.live ? grad.of(load_unit<T>(p, t, u)) : zero);
    if (p.rest)
        for (uint32_t q = w; q < p.s.nseg; q += kStreamWaves) store_any_rest<T>(p, t, q, res.live ? grad.of(any_rest<T>(p, t, q)) : zero);
    if (res.live) store_action<T, kStreamWaves>(p, t, ca, fmaf(res.coef, power_of(xa, s.top, kk), res.at_a));
}

// Rows cut into parts of kPartWaves * kPartVectors units, a workgroup to each, in two launches: the parts' statistics, then the rows'
// results, joined from them.  Where rows are few, so that all CUs share them: every workgroup joins for itself and writes its
// part of the gradient (the logits come from the caches then).  And where there is no gradient, for any number of long rows:
// nothing has to stay in registers, and many small workgroups keep more loads on their way.
constexpr int kPartWaves = 8, kPartVectors = 4, kPartUnits = kPartWaves * kPartVectors;

template <typename T> __global__ __launch_bounds__(kPartWaves * 64) void policy_part_stats_kernel(const PolicyParams p)
{
    __shared__ Stats red[kPartWaves];
    const uint32_t t = quotient(blockIdx.x, p.by_parts), part = blockIdx.x - t * p.parts, w = uniform(threadIdx.x >> 6), u0 = part * kPartUnits;
    if (!counts(p, t, action_of(p, t))) return;
    const float kk = exponent_factor(p);
    u32x4 r[kPartVectors];
#pragma unroll
    for (int i = 0; i < kPartVectors; ++i) {
        const uint32_t u = u0 + i * kPartWaves + w;
        r[i] = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
        if (u < p.units) r[i] = load_unit<T>(p, t, u);
    }
    Stats s = with_vectors<T, kPartVectors>(Stats{-INFINITY, 0.0f}, r, kk);
    if (p.rest)
        for (uint32_t q = part + w * p.parts; q < p.s.nseg; q += kPartWaves * p.parts) {
            const u32x4 v = only_own<T>(p, load_rest<T>(p, t, q));
            s = with_vectors<T, 1>(s, &v, kk);
        }
    s = group_joined<kPartWaves>(s, red, kk);
    if (threadIdx.x == 0) p.part_stats[blockIdx.x] = s;
}

// The loss of all tokens (no more than the workgroup has threads), each joined from its parts by a thread of its own, added up in
// their order
constexpr int kLossTokens = kPartWaves * 64;
template <typename T> __device__ __forceinline__ void sum_of_parts(const PolicyParams &p, float kk)
{
    __shared__ float row_loss[kLossTokens];
    const uint32_t t = threadIdx.x;
    if (t < p.tokens) {
        const int64_t a = p.wide_ids ? token_at<int64_t>(p.actions, t) : token_at<int32_t>(p.actions, t);
        float loss = 0.0f;
        if (a >= 0 && a < p.vocab && p.weight[t] != 0.0f) {
            Stats s{-INFINITY, 0.0f};
            for (uint32_t i = 0; i < p.parts; ++i) s = joined(s, p.part_stats[(size_t)t * p.parts + i], kk);
            const TokenScalars c{p.weight[t], p.old_logp[t], p.policy.kl != 0.0f ? p.ref_logp[t] : 0.0f, p.advantage[t]};
            loss = row_result(p, c, s, to_float(logit_at<T>(p, t, column_of(p, (uint32_t)a))), kk).loss;
        }
        row_loss[t] = loss;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (uint32_t i = 0; i < p.tokens; ++i) s += (double)row_loss[i];
        *p.loss = (float)s;
    }
}

// GRAD: a workgroup to a part; otherwise a wave to a token, for the scalars alone; one workgroup more for the loss
template <typename T, bool GRAD> __global__ __launch_bounds__(kPartWaves * 64) void policy_part_result_kernel(const PolicyParams p)
{
    const float kk = exponent_factor(p);
    const uint32_t t = GRAD ? quotient(blockIdx.x, p.by_parts) : blockIdx.x, part = GRAD ? blockIdx.x - t * p.parts : 0;
    if (t == p.tokens) {
        if (part == 0) sum_of_parts<T>(p, kk);
        return;
    }
    const uint32_t w = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u, u0 = part * kPartUnits;
    const int64_t a = action_of(p, t);
    const u32x4 zero = u32x4{0, 0, 0, 0};
    RowResult res{0.0f, 0.0f, 0.0f, 0.0f, false};
    Stats s{-INFINITY, 0.0f};
    Column ca{0, 0};
    float xa = 0.0f;
    u32x4 r[kPartVectors];
    if (counts(p, t, a)) {
        if constexpr (GRAD) {
#pragma unroll
            for (int i = 0; i < kPartVectors; ++i) {
                const uint32_t u = u0 + i * kPartWaves + w;
                r[i] = u < p.units ? load_unit<T>(p, t, u) : zero;
            }
        }
        ca = column_of(p, (uint32_t)a);
        xa = to_float(logit_at<T>(p, t, ca));
        for (uint32_t i = lane; i < p.parts; i += 64) s = joined(s, p.part_stats[(size_t)t * p.parts + i], kk);
        s = wave_joined(s, kk);
        res = row_result(p, scalars_of(p, t), s, xa, kk);
    }
    if (part == 0 && threadIdx.x == 0) store_scalars(p, t, res);
    if constexpr (GRAD) {
        const Gradient<T> grad(kk, s.top, res.coef);
#pragma unroll
        for (int i = 0; i < kPartVectors; ++i) {
            const uint32_t u = u0 + i * kPartWaves + w;
            if (u < p.units) store_unit<T>(p, t, u, res.live ? grad.of(r[i]) : zero);
        }
        if (p.rest)
            for (uint32_t q = part + w * p.parts; q < p.s.nseg; q += kPartWaves * p.parts)
                store_rest<T>(p, t, q, res.live ? grad.of(load_rest<T>(p, t, q)) : zero);
        if (!res.live) return;
        // the action's entry, by the thread that wrote its vector
        const uint32_t j = ca.offset / kVec<T>, unit = ca.q * p.by_ups.d + j / 64;
        const bool whole = j / 64 < p.by_ups.d;
        const uint32_t its_part = whole ? unit / kPartUnits : ca.q % p.parts, wave = whole ? unit % kPartWaves : ca.q / p.parts % kPartWaves;
        if (part != its_part || threadIdx.x != wave * 64 + (j & 63u)) return;
        store_entry<T>(p, t, ca, fmaf(res.coef, power_of(xa, s.top, kk), res.at_a));
    }
}

// The rows' losses, added up in 64 bits in an order that depends on their number alone
constexpr int kSumThreads = 512, kSumLoads = 8;
__global__ __launch_bounds__(kSumThreads) void sum_losses_kernel(const float *row_loss, uint32_t n, float *loss)
{
    __shared__ double part[kSumThreads / 64];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += kSumThreads * kSumLoads) {
        float f[kSumLoads];
#pragma unroll
        for (int k = 0; k < kSumLoads; ++k) f[k] = i + k * kSumThreads < n ? row_loss[i + k * kSumThreads] : 0.0f;
#pragma unroll
        for (int k = 0; k < kSumLoads; ++k) s += (double)f[k];
    }
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) s += wave::shfl_xor(s, m);
    if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kSumThreads / 64; ++w) s += part[w];
        *loss = (float)s;
    }
}

// How rows are walked, and what a launch needs of the workspace: the rows' losses, and the parts' statistics where rows are cut
struct Walk { Pieces s; uint32_t whole, units, rest, parts; size_t stats_at, bytes; };
constexpr int64_t kCutRows = 128, kCutParts = (int64_t(1) << 22) - 1; // rows of a gradient, and parts of all rows, up to which rows are cut
Walk walk_of(const BlockTable &X, const BlockTable &G, int64_t tokens, int64_t vocab, int dtype, bool with_dx)
{
    Walk w;
    w.s = vocab > 0 ? pieces_of(X, G, vocab, 16 / dtype_bytes(dtype)) : Pieces{1, 0, 0, 0, 0, 0};
    w.whole = (w.s.vps - (w.s.tail ? 1 : 0)) / 64;
    w.units = w.s.nseg * w.whole;
    w.rest = w.s.vps - w.whole * 64;
    // Cut rows that are worth several workgroups, where there is no gradient or whole rows would leave most CUs idle.  Cut / whole, us:
    // loss of 16 x 131072 13 / 23, 64 15 / 23, 128 24 / 25, 128 x 20000 14.5 / 14.1, 256 x 131072 41 / 34, 512 71 / 58; log probabilities of
    // 256 x 131072 18 / 30, 4096 179 / 346.
    w.parts = (tokens <= kCutRows || !with_dx) && w.units > kPartUnits ? (w.units + kPartUnits - 1) / kPartUnits : 1;
    if (tokens * w.parts > kCutParts) w.parts = 1; // (a launch holds fewer than 2^32 threads)
    w.stats_at = align_up((size_t)tokens * 4, 256);
    w.bytes = w.stats_at + (w.parts > 1 ? align_up((size_t)tokens * w.parts * sizeof(Stats), 256) : 0);
    return w;
}

// What covers any smaller number of tokens too: rows are cut where they are few, and need more then.
size_t room_of(const BlockTable &X, const BlockTable &G, int64_t tokens, int64_t vocab, int dtype, bool with_dx)
{
    const Walk w = walk_of(X, G, tokens, vocab, dtype, with_dx);
    const int64_t parts = (w.units + kPartUnits - 1) / kPartUnits, cut = std::min({tokens, with_dx ? kCutRows : tokens, kCutParts / std::max<int64_t>(parts, 1)});
    return std::max(w.bytes, walk_of(X, G, cut, vocab, dtype, with_dx).bytes);
}

// workgroups that fit the chip at a time: on each of 256 CUs 16 waves of up to 128 registers, or 32 of those that hold a few vectors
template <typename T, int WAVES, int NC, bool GRAD> void launch_rows(PolicyParams &p, hipStream_t s)
{
    const uint32_t most = 256 * (NC <= 4 && WAVES < 16 ? 32 : 16) / WAVES;
    p.groups = p.tokens < most ? p.tokens : most;
    hipLaunchKernelGGL((policy_rows_kernel<T, WAVES, NC, GRAD>), dim3(p.groups), dim3(WAVES * 64), 0, s, p);
}

template <typename T> tt_status launch_policy(PolicyParams &p, hipStream_t s)
{
    const uint32_t u = p.units, q = p.rest ? p.s.nseg : 0; // whole units, and segments with a rest: one at most to a wave, a vector at least
    const auto fits = [&](uint32_t waves, uint32_t nc) { return u <= waves * nc && q <= waves && p.s.seg >= (uint32_t)kVec<T>; };
    bool summed = !p.loss;
    if (p.parts > 1) {
        // (a workgroup of the second launch has a thread per token for the loss)
        const uint32_t one_more = p.loss && p.tokens <= (p.with_dx ? (uint32_t)kLossTokens : 64u) ? 1 : 0;
        summed = summed || one_more;
        hipLaunchKernelGGL((policy_part_stats_kernel<T>), dim3(p.tokens * p.parts), dim3(kPartWaves * 64), 0, s, p);
        if (p.with_dx) hipLaunchKernelGGL((policy_part_result_kernel<T, true>), dim3((p.tokens + one_more) * p.parts), dim3(kPartWaves * 64), 0, s, p);
        else hipLaunchKernelGGL((policy_part_result_kernel<T, false>), dim3(p.tokens + one_more), dim3(64), 0, s, p);
    } else if (!fits(16, p.with_dx ? 20 : 2)) {
        hipLaunchKernelGGL((policy_stream_kernel<T>), dim3(p.tokens), dim3(kStreamWaves * 64), 0, s, p);
    } else if (!p.with_dx) {
        if (p.tokens <= 256) {
            if (fits(4, 1)) launch_rows<T, 4, 1, false>(p, s);
            else launch_rows<T, 16, 2, false>(p, s);
        } else {
            if (fits(1, 4)) launch_rows<T, 1, 4, false>(p, s);
            else if (fits(4, 8)) launch_rows<T, 4, 8, false>(p, s);
            else launch_rows<T, 16, 2, false>(p, s);
        }
    } else if (p.tokens <= 256) { // a CU to every row: as many waves as have something to do (200 x 32768 14.2 us, by the next rule 15.8)
        if (fits(4, 1)) launch_rows<T, 4, 1, true>(p, s);
        else if (fits(16, 2)) launch_rows<T, 16, 2, true>(p, s);
        else if (fits(16, 4)) launch_rows<T, 16, 4, true>(p, s);
        else if (fits(16, 8)) launch_rows<T, 16, 8, true>(p, s);
        else if (fits(16, 16)) launch_rows<T, 16, 16, true>(p, s);
        else launch_rows<T, 16, 20, true>(p, s);
    } else {
        if (fits(1, 1)) launch_rows<T, 1, 1, true>(p, s);
        else if (fits(1, 2)) launch_rows<T, 1, 2, true>(p, s);
        else if (fits(1, 4)) launch_rows<T, 1, 4, true>(p, s);
        else if (fits(1, 8)) launch_rows<T, 1, 8, true>(p, s);
        else if (fits(1, 16)) launch_rows<T, 1, 16, true>(p, s);
        else if (fits(2, 16)) launch_rows<T, 2, 16, true>(p, s);
        else if (fits(4, 16)) launch_rows<T, 4, 16, true>(p, s);
        else if (fits(8, 16)) launch_rows<T, 8, 16, true>(p, s);
        else if (fits(16, 16)) launch_rows<T, 16, 16, true>(p, s);
        else launch_rows<T, 16, 20, true>(p, s);
    }
    if (!summed) hipLaunchKernelGGL(sum_losses_kernel, dim3(1), dim3(kSumThreads), 0, s, p.row_loss, p.tokens, p.loss);
    return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
}

tt_status launch_policy(PolicyParams &p, const Walk &w, void *workspace, int dtype, int id_dtype, hipStream_t s)
{
    p.wide_ids = id_dtype == TT_I64;
    p.s = w.s;
    p.by_ups = divisor(w.whole ? w.whole : 1);
    p.by_ups.d = w.whole;
    p.units = w.units;
    p.rest = w.rest;
    p.parts = w.parts;
    p.by_parts = divisor(w.parts);
    p.part_stats = reinterpret_cast<Stats *>(static_cast<char *>(workspace) + w.stats_at);
    return dtype == TT_BF16 ? launch_policy<uint16_t>(p, s) : launch_policy<float>(p, s);
}

tt_status check_sizes(int64_t tokens, int64_t vocab, int k, int dtype, const tt_tiling &tX)
{
    if (!valid_k(k) || !valid_tiling(tX, k) || !valid_dtype(dtype) || tokens < 0 || vocab < 0) return TT_EINVAL;
    // a launch holds fewer than 2^32 threads, a workgroup per token
    if (tokens >= (int64_t(1) << 22) || !fits31(vocab)) return TT_EUNSUPPORTED;
    return TT_OK;
}

} // namespace
} // namespace tt

extern "C" tt_status tt_policy_workspace_bytes(int64_t tokens, int64_t vocab, int k, int dtype, tt_tiling tX, tt_tiling tdX,
                                               int with_dx, size_t *bytes)
{
    using namespace tt;
    if (!bytes) return TT_EINVAL;
    tt_status st = check_sizes(tokens, vocab, k, dtype, tX);
    if (st != TT_OK) return st;
    if (with_dx && !valid_tiling(tdX, k)) return TT_EINVAL;
    BlockTable X, G;
    if (!make_blocks(nullptr, tX, k, tokens, vocab, &X)) return TT_EINFEASIBLE;
    G = X;
    if (with_dx && !make_blocks(nullptr, tdX, k, tokens, vocab, &G)) return TT_EINFEASIBLE;
    *bytes = room_of(X, G, tokens, vocab, dtype, with_dx != 0);
    return TT_OK;
}

extern "C" tt_status tt_policy_loss(const tt_policy *policy, int64_t tokens, int64_t vocab, int k, int dtype, tt_tiling tX, tt_tiling tdX,
                                    const void *const *X, int id_dtype, const void *actions, const float *old_logp,
                                    const float *ref_logp, const float *advantage, const float *weight, float *loss, float *logp,
                                    void *const *dX, void *workspace, size_t ws_bytes, void *stream)
{
    using namespace tt;
    tt_status st = check_sizes(tokens, vocab, k, dtype, tX);
    if (st != TT_OK) return st;
    if (!policy || !(policy->scale > 0.0f) || std::isinf(policy->scale) || !(policy->clip_low >= 0.0f) || !(policy->clip_high >= 0.0f) ||
        std::isnan(policy->kl) || std::isinf(policy->kl))
        return TT_EINVAL;
    const int e = dtype_bytes(dtype);
    const bool empty = tokens == 0 || vocab == 0;
    if (!shards_fit(X, k, e, empty) || (dX && (!valid_tiling(tdX, k) || !shards_fit(const_cast<const void *const *>(dX), k, e, empty)))) return TT_EINVAL;
    if ((id_dtype != TT_I32 && id_dtype != TT_I64) || !aligned_to(loss, 4)) return TT_EINVAL;
    if (tokens > 0 && (!aligned_to(actions, id_dtype == TT_I32 ? 4 : 8) || !aligned_to(old_logp, 4) || !aligned_to(advantage, 4) || !aligned_to(weight, 4) ||
                       (policy->kl != 0.0f && !aligned_to(ref_logp, 4)) || (logp && !aligned_to(logp, 4))))
        return TT_EINVAL;
    PolicyParams p;
    if (!make_blocks(X, tX, k, tokens, vocab, &p.X)) return TT_EINFEASIBLE;
    p.G = p.X;
    p.with_dx = dX != nullptr;
    if (dX && !make_blocks(const_cast<const void *const *>(dX), tdX, k, tokens, vocab, &p.G)) return TT_EINFEASIBLE;
    const Walk w = walk_of(p.X, p.G, tokens, vocab, dtype, p.with_dx != 0);
    if (tokens > 0 && (!workspace || ws_bytes < w.bytes || reinterpret_cast<uintptr_t>(workspace) % 256)) return TT_EWORKSPACE;
    p.actions = actions;
    p.old_logp = old_logp;
    p.ref_logp = ref_logp;
    p.advantage = advantage;
    p.weight = weight;
    p.logp = logp;
    p.row_loss = static_cast<float *>(workspace);
    p.tokens = (uint32_t)tokens;
    p.vocab = vocab;
    p.policy = *policy;
    const uint64_t all = (uint64_t)tokens * (uint64_t)vocab * e;
    ProfileScope scope(stream, TT_K_LOSS, 1 << k, tokens, vocab, e, all * (1 + (dX ? p.G.nrep : 0)), 0);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    p.loss = loss;
    if (tokens > 0) return launch_policy(p, w, workspace, dtype, id_dtype, s);
    hipLaunchKernelGGL(sum_losses_kernel, dim3(1), dim3(kSumThreads), 0, s, p.row_loss, p.tokens, loss);
    return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
}

extern "C" tt_status tt_token_logp(int64_t tokens, int64_t vocab, int k, int dtype, tt_tiling tX, float scale, const void *const *X,
                                   int id_dtype, const void *ids, float *logp, void *workspace, size_t ws_bytes, void *stream)
{
    using namespace tt;
    tt_status st = check_sizes(tokens, vocab, k, dtype, tX);
    if (st != TT_OK) return st;
    const int e = dtype_bytes(dtype);
    if (!(scale > 0.0f) || std::isinf(scale) || !shards_fit(X, k, e, tokens == 0 || vocab == 0) || (id_dtype != TT_I32 && id_dtype != TT_I64)) return TT_EINVAL;
    if (tokens > 0 && (!aligned_to(ids, id_dtype == TT_I32 ? 4 : 8) || !aligned_to(logp, 4))) return TT_EINVAL;
    PolicyParams p;
    if (!make_blocks(X, tX, k, tokens, vocab, &p.X)) return TT_EINFEASIBLE;
    if (tokens == 0) return TT_OK;
    p.G = p.X;
    p.with_dx = 0;
    const Walk w = walk_of(p.X, p.G, tokens, vocab, dtype, p.with_dx != 0);
    if (!workspace || ws_bytes < w.bytes || reinterpret_cast<uintptr_t>(workspace) % 256) return TT_EWORKSPACE;
    p.actions = ids;
    p.old_logp = p.ref_logp = p.advantage = p.weight = nullptr;
    p.logp = logp;
    p.row_loss = p.loss = nullptr;
    p.tokens = (uint32_t)tokens;
    p.vocab = vocab;
    p.policy = tt_policy{scale, 0.0f, 0.0f, 0.0f};
    ProfileScope scope(stream, TT_K_LOSS, 1 << k, tokens, vocab, e, (uint64_t)tokens * (uint64_t)vocab * e, 0);
    return launch_policy(p, w, workspace, dtype, id_dtype, reinterpret_cast<hipStream_t>(stream));
}
