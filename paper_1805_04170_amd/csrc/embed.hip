// Embedding of tokens and its table's gradient, on tiled tensors: the rows of a table by token number in front of a chain of
// layers, and the sum of the rows' gradients by token number behind its backward pass.
//
// Both move rows and hardly compute: what bounds them is memory (the result is written once, every row read once) and, for a
// few tokens, the trip to a token's number and on to its row.
#include <cstdint>
#include <type_traits>
#include "launch_util.h"
#include "block_table.h"
#include "tensor_tiling_tokens.h"
#include "tiled_rows.h"

namespace tt {
namespace {

constexpr int kThreads = 256;
constexpr int kU = 4; // vectors per lane and unit of work

// A unit of work is kU vectors per lane of a group of lanes; a row is `upr` units.
struct RowSplit : Pieces {
    uint32_t upr;  // units per row
    uint32_t glog; // log2 of the lanes of a group
};

RowSplit split_row(const BlockTable &a, const BlockTable &b, int64_t cols, int ev)
{
    RowSplit s;
    static_cast<Pieces &>(s) = pieces_of(a, b, cols, ev);
    s.glog = 0;
    while (s.glog < 6 && (1u << s.glog) < s.nvec) ++s.glog;
    s.upr = (s.nvec + (kU << s.glog) - 1) / (kU << s.glog);
    return s;
}

// ------------------------------------------------------------------------------------------------------- forward

struct EmbedParams {
    BlockTable W, X;
    RowSplit s;
    const void *ids;
    uint32_t tokens, units;
    int64_t vocab;
    float scale;
};

// One unit per group of lanes: kU vectors of one token's row, all of them loaded before the first is stored.
template <typename T, typename I> __global__ __launch_bounds__(kThreads) void embed_forward_kernel(const EmbedParams p)
{
    const uint32_t g = (blockIdx.x * kThreads + threadIdx.x) >> p.s.glog, l = threadIdx.x & ((1u << p.s.glog) - 1);
    if (g >= p.units) return;
    const uint32_t t = g / p.s.upr, j0 = ((g - t * p.s.upr) * kU << p.s.glog) + l;
    const int64_t v = token_at<I>(p.ids, t);
    const bool in = v >= 0 && v < p.vocab;
    u32x4 r[kU];
    uint32_t col[kU], n[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const uint32_t j = j0 + ((uint32_t)u << p.s.glog);
        r[u] = u32x4{0, 0, 0, 0};
        n[u] = 0;
        if (j < p.s.nvec) {
            vector_of(p.s, kVec<T>, j, &col[u], &n[u]);
            if (in) r[u] = load_vector(source_of<T>(p.W, (uint32_t)v, col[u]), n[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        if (n[u] == 0) continue;
        float f[kVec<T>];
        unpack16(r[u], f, T());
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) f[i] = in ? f[i] * p.scale : 0.0f;
        store_all<T>(p.X, t, col[u], n[u], pack16(f, T()));
    }
}

// ------------------------------------------------------------------------------------------------------ backward
// Three launches.  (1) Tokens sorted by number, stably: `order` lists the tokens with number 0, then 1, ...; `start[v]` is
// where v's begin.  (2) Numbers with many tokens (more than `chunk`) would keep one group of lanes busy long after the
// rest is done: the sorted list is cut into runs of `chunk`, and each run adds up its part of such a number into a
// partial sum.  (3) Every row of the table's gradient: the sum over its tokens in order, or over its partial sums.

// (1) A workgroup owns a range of numbers and reads all tokens, each wave a stretch of them: it counts how many lie below its
// range (where its part of the list begins) and how often each of its numbers comes in each wave's stretch; after a scan
// over (number, wave) the waves walk their stretches again and put their tokens in place, in order.  No workgroup waits for
// another, whatever the numbers are.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortRange = 1024;

struct SortParams {
    const void *ids;
    uint32_t tokens, range; // numbers per workgroup
    int64_t vocab;
    uint32_t *order, *start;
};

template <typename I> __global__ __launch_bounds__(kSortThreads) void sort_tokens_kernel(const SortParams p)
{
    __shared__ uint32_t at[kSortWaves * kSortRange];
    __shared__ uint32_t part[kSortWaves + 1];
    const uint32_t lane = threadIdx.x & 63u, w = uniform(threadIdx.x >> 6);
    const int64_t lo = (int64_t)blockIdx.x * p.range;
    const uint32_t own = (uint32_t)(p.vocab - lo < (int64_t)p.range ? p.vocab - lo : (int64_t)p.range);
    for (uint32_t i = threadIdx.x; i < kSortWaves * p.range; i += kSortThreads) at[i] = 0;
    __syncthreads();
    const uint32_t stretch = ((p.tokens + kSortThreads - 1) / kSortThreads) * 64;
    const uint32_t t0 = w * stretch < p.tokens ? w * stretch : p.tokens, t1 = t0 + stretch < p.tokens ? t0 + stretch : p.tokens;
    uint32_t *mine = at + w * p.range;
    uint32_t below = 0;
    for (uint32_t t = t0 + lane; t < t1; t += 64) {
        const int64_t v = token_at<I>(p.ids, t);
        if (v >= 0 && v < lo) ++below;
        if (v >= lo && v < lo + own) wave::lds_add(&mine[v - lo], 1);
    }
    below = wave_sum(below);
    if (lane == 0) part[w] = below;
    __syncthreads();
    // thread r: number lo + r; exclusive scan of the totals over the workgroup
    uint32_t total = 0, base = 0;
    if (threadIdx.x < own)
        for (uint32_t i = 0; i < (uint32_t)kSortWaves; ++i) total += at[i * p.range + threadIdx.x];
    for (uint32_t i = 0; i < (uint32_t)kSortWaves; ++i) base += part[i];
    uint32_t incl = total;
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
        const uint32_t o = wave::shfl_up(incl, by);
        if (lane >= (uint32_t)by) incl += o;
    }
    __syncthreads();
    if (lane == 63) part[w] = incl;
    __syncthreads();
    uint32_t before = base + incl - total;
    for (uint32_t i = 0; i < w; ++i) before += part[i];
    if (threadIdx.x < own) {
        p.start[lo + threadIdx.x] = before;
        uint32_t run = before;
        for (uint32_t i = 0; i < (uint32_t)kSortWaves; ++i) {
            const uint32_t c = at[i * p.range + threadIdx.x];
            at[i * p.range + threadIdx.x] = run;
            run += c;
        }
        if (lo + threadIdx.x + 1 == p.vocab) p.start[p.vocab] = run;
    }
    __syncthreads();
    for (uint32_t tt0 = t0; tt0 < t1; tt0 += 64) {
        const uint32_t t = tt0 + lane;
        const int64_t v = t < t1 ? token_at<I>(p.ids, t) : -1;
        const bool in = v >= lo && v < lo + own;
        const uint32_t r = in ? (uint32_t)(v - lo) : 0;
        uint64_t left = wave::ballot(in);
        while (left) { // one number of the 64 tokens at a time
            const uint32_t n = wave::read_lane(r, __builtin_ctzll(left));
            const bool same = in && r == n;
            const uint64_t who = wave::ballot(same);
            const uint32_t to = mine[n];
            wave::fence();
            if (same) {
                const uint32_t rank = (uint32_t)__builtin_popcountll(who & ((uint64_t(1) << lane) - 1));
                p.order[to + rank] = t;
                if (rank == 0) mine[n] = to + (uint32_t)__builtin_popcountll(who);
            }
            wave::fence();
            left &= ~who;
        }
    }
}

struct EmbedGradParams {
    BlockTable G, W; // the rows' gradients, the table's
    RowSplit s;
    const void *ids;
    const uint32_t *order, *start;
    float *partial; // [2 runs][cols]: run c's part of a number that began before the run, of one that begins inside it
    uint32_t chunk, runs, cols, units;
    int64_t vocab;
    float scale;
};

template <typename T> struct Sums {
    float f[kU][kVec<T>];
    uint32_t col[kU], n[kU];
};

template <typename T> __device__ __forceinline__ void begin(Sums<T> &a, const RowSplit &s, uint32_t j0)
{
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const uint32_t j = j0 + ((uint32_t)u << s.glog);
        a.n[u] = 0;
        a.col[u] = 0;
        if (j < s.nvec) vector_of(s, kVec<T>, j, &a.col[u], &a.n[u]);
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) a.f[u][i] = 0.0f;
    }
}

// the rows order[b .. e) added to the sums, in that order
template <typename T> __device__ __forceinline__ void add_rows(Sums<T> &a, const EmbedGradParams &p, uint32_t b, uint32_t e)
{
    for (uint32_t i = b; i < e; ++i) {
        const uint32_t t = p.order[i];
        u32x4 r[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            r[u] = u32x4{0, 0, 0, 0};
            if (a.n[u]) r[u] = load_vector(source_of<T>(p.G, t, a.col[u]), a.n[u]);
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            float f[kVec<T>];
            unpack16(r[u], f, T());
#pragma unroll
            for (int q = 0; q < kVec<T>; ++q) a.f[u][q] += f[q];
        }
    }
}

// (2)
template <typename T, typename I> __global__ __launch_bounds__(kThreads) void embed_runs_kernel(const EmbedGradParams p)
{
    const uint32_t g = (blockIdx.x * kThreads + threadIdx.x) >> p.s.glog, l = threadIdx.x & ((1u << p.s.glog) - 1);
    if (g >= p.units) return;
    const uint32_t c = g / p.s.upr, j0 = ((g - c * p.s.upr) * kU << p.s.glog) + l;
    const uint32_t total = p.start[p.vocab];
    const uint32_t b = c * p.chunk;
    if (b >= total) return;
    const uint32_t e = b + p.chunk < total ? b + p.chunk : total;
    const int64_t first = token_at<I>(p.ids, p.order[b]), last = token_at<I>(p.ids, p.order[e - 1]);
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const int64_t v = side == 0 ? first : last;
        if (side == 1 && last == first) break;
        const uint32_t vb = p.start[v], ve = p.start[v + 1];
        if (ve - vb <= p.chunk) continue; // (a number with more tokens than a run holds reaches the run's first or last place)
        Sums<T> a;
        begin(a, p.s, j0);
        add_rows(a, p, vb > b ? vb : b, ve < e ? ve : e);
        float *to = p.partial + (size_t)(2 * c + (vb > b ? 1 : 0)) * p.cols;
#pragma unroll
        for (int u = 0; u < kU; ++u)
            for (uint32_t i = 0; i < a.n[u]; ++i) to[a.col[u] + i] = a.f[u][i];
    }
}

// (3)
template <typename T> __global__ __launch_bounds__(kThreads) void embed_rows_kernel(const EmbedGradParams p)
{
    const uint64_t g = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) >> p.s.glog;
    const uint32_t l = threadIdx.x & ((1u << p.s.glog) - 1);
    const uint64_t row = g / p.s.upr;
    if (row >= (uint64_t)p.vocab) return;
    const uint32_t v = (uint32_t)row, j0 = ((uint32_t)(g - row * p.s.upr) * kU << p.s.glog) + l;
    const uint32_t b = p.start[v], e = p.start[v + 1];
    Sums<T> a;
    begin(a, p.s, j0);
    if (e - b <= p.chunk) {
        add_rows(a, p, b, e);
    } else {
        for (uint32_t c = b / p.chunk; c * p.chunk < e; ++c) {
            const float *from = p.partial + (size_t)(2 * c + (b > c * p.chunk ? 1 : 0)) * p.cols;
#pragma unroll
            for (int u = 0; u < kU; ++u)
                for (uint32_t i = 0; i < a.n[u]; ++i) a.f[u][i] += from[a.col[u] + i];
        }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        if (a.n[u] == 0) continue;
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) a.f[u][i] *= p.scale;
        store_all<T>(p.W, v, a.col[u], a.n[u], pack16(a.f[u], T()));
    }
}

// ----------------------------------------------------------------------------------------------------- host side

tt_status check_sizes(int64_t tokens, int64_t vocab, int64_t width, int k, int dtype, const tt_tiling &a, const tt_tiling &b)
{
    if (!valid_k(k) || !valid_tiling(a, k) || !valid_tiling(b, k) || !valid_dtype(dtype)) return TT_EINVAL;
    if (tokens < 0 || vocab < 0 || width < 0) return TT_EINVAL;
    if (!fits31(tokens) || !fits31(vocab) || !fits31(width)) return TT_EUNSUPPORTED;
    return TT_OK;
}

bool valid_ids(int id_dtype, const void *ids, int64_t tokens)
{
    if (id_dtype != TT_I32 && id_dtype != TT_I64) return false;
    return tokens == 0 || aligned_to(ids, id_dtype == TT_I32 ? 4 : 8);
}

// places of the sorted list per run: a run is added up by one group of lanes and the runs of a number by another, so both are
// to stay short
uint32_t run_length(int64_t tokens) { return tokens <= 8192 ? 32 : tokens <= 65536 ? 64 : 128; }

struct GradSpace {
    size_t order, start, partial, bytes;
    uint32_t runs;
};
GradSpace grad_space(int64_t tokens, int64_t vocab, int64_t width)
{
    GradSpace s;
    const uint32_t chunk = run_length(tokens);
    s.runs = tokens > chunk ? (uint32_t)((tokens + chunk - 1) / chunk) : 0;
    s.order = 0;
    s.start = align_up((size_t)tokens * 4, 256);
    s.partial = s.start + align_up(((size_t)vocab + 1) * 4, 256);
    s.bytes = s.partial + align_up((size_t)2 * s.runs * (size_t)width * 4, 256);
    return s;
}

tt_status launched() { return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE; }

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
    if (!valid_ids(id_dtype, ids, tokens) || !shards_fit(W, k, e) || !shards_fit(const_cast<const void *const *>(X), k, e)) return TT_EINVAL;
    EmbedParams p;
    if (!make_blocks(W, tW, k, vocab, width, &p.W) || !make_blocks(const_cast<const void *const *>(X), tX, k, tokens, width, &p.X)) return TT_EINFEASIBLE;
    if (tokens == 0 || width == 0) return TT_OK;
    p.s = split_row(p.W, p.X, width, 16 / e);
    p.ids = ids;
    p.tokens = (uint32_t)tokens;
    p.vocab = vocab;
    p.scale = scale;
    const uint64_t units = (uint64_t)tokens * p.s.upr, groups = (uint64_t)kThreads >> p.s.glog, grid = (units + groups - 1) / groups;
    if (grid * kThreads >= (uint64_t(1) << 32)) return TT_EUNSUPPORTED;
    p.units = (uint32_t)units;
    const uint64_t row = (uint64_t)width * e;
    ProfileScope scope(stream, TT_K_EMBED, 1 << k, tokens, width, e, (uint64_t)tokens * row * (1 + p.X.nrep), 0);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const dim3 g((uint32_t)grid), b(kThreads);
    if (dtype == TT_BF16) {
        if (id_dtype == TT_I32) hipLaunchKernelGGL((embed_forward_kernel<uint16_t, int32_t>), g, b, 0, s, p);
        else hipLaunchKernelGGL((embed_forward_kernel<uint16_t, int64_t>), g, b, 0, s, p);
    } else {
        if (id_dtype == TT_I32) hipLaunchKernelGGL((embed_forward_kernel<float, int32_t>), g, b, 0, s, p);
        else hipLaunchKernelGGL((embed_forward_kernel<float, int64_t>), g, b, 0, s, p);
    }
    return launched();
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
    *bytes = grad_space(tokens, vocab, width).bytes;
    return TT_OK;
}

namespace tt {
namespace {

template <typename T, typename I>
tt_status launch_embed_grad(const SortParams &sp, EmbedGradParams &p, uint32_t sort_groups, uint32_t run_groups, uint32_t row_groups, hipStream_t s)
{
    hipLaunchKernelGGL((sort_tokens_kernel<I>), dim3(sort_groups), dim3(kSortThreads), 0, s, sp);
    if (run_groups) hipLaunchKernelGGL((embed_runs_kernel<T, I>), dim3(run_groups), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL((embed_rows_kernel<T>), dim3(row_groups), dim3(kThreads), 0, s, p);
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
    if (!valid_ids(id_dtype, ids, tokens) || !shards_fit(dX, k, e) || !shards_fit(const_cast<const void *const *>(dW), k, e)) return TT_EINVAL;
    EmbedGradParams p;
    if (!make_blocks(dX, tdX, k, tokens, width, &p.G) || !make_blocks(const_cast<const void *const *>(dW), tdW, k, vocab, width, &p.W)) return TT_EINFEASIBLE;
    if (vocab == 0 || width == 0) return TT_OK;
    const GradSpace sp = grad_space(tokens, vocab, width);
    if (!workspace || ws_bytes < sp.bytes || reinterpret_cast<uintptr_t>(workspace) % 256) return TT_EWORKSPACE;
    char *ws = static_cast<char *>(workspace);
    SortParams q;
    q.ids = ids;
    q.tokens = (uint32_t)tokens;
    q.vocab = vocab;
    // a range of numbers per CU, at most what a workgroup's counters hold
    const int64_t per_cu = (vocab + 255) / 256;
    q.range = (uint32_t)(per_cu < kSortRange ? per_cu : kSortRange);
    q.order = reinterpret_cast<uint32_t *>(ws + sp.order);
    q.start = reinterpret_cast<uint32_t *>(ws + sp.start);
    const uint32_t sort_groups = (uint32_t)((vocab + q.range - 1) / q.range);
    p.s = split_row(p.G, p.W, width, 16 / e);
    p.ids = ids;
    p.order = q.order;
    p.start = q.start;
    p.partial = reinterpret_cast<float *>(ws + sp.partial);
    p.chunk = run_length(tokens);
    p.runs = sp.runs;
    p.cols = (uint32_t)width;
    p.vocab = vocab;
    p.scale = scale;
    const uint64_t groups = (uint64_t)kThreads >> p.s.glog;
    const uint64_t run_units = (uint64_t)sp.runs * p.s.upr, run_groups = (run_units + groups - 1) / groups;
    const uint64_t row_groups = ((uint64_t)vocab * p.s.upr + groups - 1) / groups;
    if (run_groups * kThreads >= (uint64_t(1) << 32) || row_groups * kThreads >= (uint64_t(1) << 32)) return TT_EUNSUPPORTED;
    p.units = (uint32_t)run_units;
    const uint64_t row = (uint64_t)width * e;
    ProfileScope scope(stream, TT_K_EMBED_GRAD, 1 << k, vocab, width, e, (uint64_t)tokens * row + (uint64_t)vocab * row * p.W.nrep, 0);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const uint32_t rg = (uint32_t)run_groups, wg = (uint32_t)row_groups;
    if (dtype == TT_BF16)
        return id_dtype == TT_I32 ? launch_embed_grad<uint16_t, int32_t>(q, p, sort_groups, rg, wg, s)
                                  : launch_embed_grad<uint16_t, int64_t>(q, p, sort_groups, rg, wg, s);
    return id_dtype == TT_I32 ? launch_embed_grad<float, int32_t>(q, p, sort_groups, rg, wg, s)
                              : launch_embed_grad<float, int64_t>(q, p, sort_groups, rg, wg, s);
}
