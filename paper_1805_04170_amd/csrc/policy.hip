// The clipped policy loss on a chain's logits and its gradient, and the tokens' log probabilities alone.
//
// A row of logits gives one number, log p[a] = z_a - log sum exp z, and with its derivative g of the loss the row's gradient
// g (onehot(a) - p): two sums over the row and a pass that writes as much as was read.  Memory bounds it (8 flops and two
// exponentials a value), so the logits are to come from memory once.
#include <cmath>
#include <cstdint>
#include "launch_util.h"
#include "tiled_rows.h"

namespace tt {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PolicyParams {
    BlockTable X, G;
    Pieces s;
    const void *actions;
    const float *old_logp, *ref_logp, *advantage, *weight; // weight NULL: log probabilities alone
    float *logp, *row_loss;                                // either may be NULL
    uint32_t tokens;
    int64_t vocab;
    tt_policy policy;
};

// What a row's statistics come to: its log probability, its part of the loss, and the derivative by the log probability
struct RowLoss { float logp, loss, d; };

__device__ __forceinline__ RowLoss row_loss(const PolicyParams &p, uint32_t t, float logp)
{
    RowLoss r{logp, 0.0f, 0.0f};
    if (!p.weight) return r;
    const float w = p.weight[t], adv = p.advantage[t], lo = 1.0f - p.policy.clip_low, hi = 1.0f + p.policy.clip_high;
    const float ratio = expf(logp - p.old_logp[t]);
    const float clipped = ratio < lo ? lo : ratio > hi ? hi : ratio;
    const float a = ratio * adv, b = clipped * adv;
    r.loss = a < b || a != a ? -a : -b;
    const bool held = (adv > 0.0f && ratio > hi) || (adv < 0.0f && ratio < lo);
    r.d = held ? 0.0f : -a;
    if (p.policy.kl != 0.0f) {
        const float diff = p.ref_logp[t] - logp, em1 = expm1f(diff);
        r.loss += p.policy.kl * (em1 - diff);
        r.d -= p.policy.kl * em1;
    }
    r.loss *= w;
    r.d *= w;
    return r;
}

// Over a workgroup of WAVES waves; every thread gets the result.  `red` is WAVES floats that no earlier reader still needs.
template <int WAVES> __device__ __forceinline__ float group_max(float v, float *red)
{
    v = wave_max(v);
    if constexpr (WAVES == 1) return v;
    if ((threadIdx.x & 63u) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v = fmaxf(v, red[i]);
    return v;
}
template <int WAVES> __device__ __forceinline__ float group_sum(float v, float *red)
{
    v = wave_sum(v);
    if constexpr (WAVES == 1) return v;
    if ((threadIdx.x & 63u) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v += red[i];
    return v;
}

// One workgroup per token; the row is read for its maximum, for its sum and for its gradient (the later times from the caches,
// where it fits).
template <typename T, typename I, int THREADS> __global__ __launch_bounds__(THREADS) void policy_stream_kernel(const PolicyParams p)
{
    constexpr int EV = kVec<T>, WAVES = THREADS / 64;
    __shared__ float red[2][WAVES];
    const uint32_t t = blockIdx.x;
    const int64_t a = token_at<I>(p.actions, t);
    const bool in = a >= 0 && a < p.vocab && !(p.weight && p.weight[t] == 0.0f);
    const float kk = p.policy.scale * kLog2e;
    RowLoss r{0.0f, 0.0f, 0.0f};
    float top = 0.0f, coef = 0.0f;
    bool live = false;
    if (in) {
        float m = -INFINITY;
        for (uint32_t j = threadIdx.x; j < p.s.nvec; j += THREADS) {
            uint32_t col, n;
            vector_of(p.s, EV, j, &col, &n);
            float f[EV];
            unpack16(load_vector(source_of<T>(p.X, t, col), n), f, T());
#pragma unroll
            for (int i = 0; i < EV; ++i) m = (uint32_t)i < n ? fmaxf(m, f[i]) : m;
        }
        m = group_max<WAVES>(m, red[0]);
        top = m * kk;
        const bool bottom = m == -INFINITY; // nothing above -inf: all -inf, or NaN among them
        float s = 0.0f;
        for (uint32_t j = threadIdx.x; j < p.s.nvec; j += THREADS) {
            uint32_t col, n;
            vector_of(p.s, EV, j, &col, &n);
            float f[EV];
            unpack16(load_vector(source_of<T>(p.X, t, col), n), f, T());
#pragma unroll
            for (int i = 0; i < EV; ++i) {
                const float e = bottom ? (f[i] == -INFINITY ? 0.0f : f[i]) : wave::exp2_fast(fmaf(f[i], kk, -top));
                s += (uint32_t)i < n ? e : 0.0f;
            }
        }
        s = group_sum<WAVES>(s, red[1]);
        live = !(bottom && s == 0.0f);
        if (live) {
            const float xa = to_float(*source_of<T>(p.X, t, (uint32_t)a));
            r = row_loss(p, t, (fmaf(xa, kk, -top) - log2f(s)) * kLn2);
            coef = -r.d * p.policy.scale / s;
        }
    }
    if (threadIdx.x == 0) {
        if (p.logp) p.logp[t] = r.logp;
        if (p.row_loss) p.row_loss[t] = r.loss;
    }
    if (!p.G.p[0]) return;
    const float at_a = r.d * p.policy.scale;
    for (uint32_t j = threadIdx.x; j < p.s.nvec; j += THREADS) {
        uint32_t col, n;
        vector_of(p.s, EV, j, &col, &n);
        float f[EV];
        if (live) {
            unpack16(load_vector(source_of<T>(p.X, t, col), n), f, T());
#pragma unroll
            for (int i = 0; i < EV; ++i) {
                f[i] = coef * wave::exp2_fast(fmaf(f[i], kk, -top));
                if ((int64_t)col + i == a) f[i] += at_a;
            }
        } else {
#pragma unroll
            for (int i = 0; i < EV; ++i) f[i] = 0.0f;
        }
        store_all<T>(p.G, t, col, n, pack16(f, T()));
    }
}

// The rows' losses, added up in an order that depends on their number alone
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void sum_losses_kernel(const float *row_loss, uint32_t n, float *loss)
{
    __shared__ float red[kSumThreads / 64];
    float s = 0.0f;
    for (uint32_t i = threadIdx.x; i < n; i += kSumThreads) s += row_loss[i];
    s = group_sum<kSumThreads / 64>(s, red);
    if (threadIdx.x == 0) *loss = s;
}

size_t policy_space(int64_t tokens) { return align_up((size_t)tokens * 4, 256); }

template <typename T, typename I> tt_status launch_policy(const PolicyParams &p, hipStream_t s)
{
    if (p.vocab >= 8192) hipLaunchKernelGGL((policy_stream_kernel<T, I, 1024>), dim3(p.tokens), dim3(1024), 0, s, p);
    else hipLaunchKernelGGL((policy_stream_kernel<T, I, 256>), dim3(p.tokens), dim3(256), 0, s, p);
    return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
}

tt_status launch_policy(const PolicyParams &p, int dtype, int id_dtype, hipStream_t s)
{
    if (dtype == TT_BF16) return id_dtype == TT_I32 ? launch_policy<uint16_t, int32_t>(p, s) : launch_policy<uint16_t, int64_t>(p, s);
    return id_dtype == TT_I32 ? launch_policy<float, int32_t>(p, s) : launch_policy<float, int64_t>(p, s);
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
    Grid g;
    if (!make_grid(tX.cut, k, tokens, vocab, &g) || (with_dx && !make_grid(tdX.cut, k, tokens, vocab, &g))) return TT_EINFEASIBLE;
    *bytes = policy_space(tokens);
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
    if (!shards_fit(X, k, e) || (dX && (!valid_tiling(tdX, k) || !shards_fit(const_cast<const void *const *>(dX), k, e)))) return TT_EINVAL;
    if ((id_dtype != TT_I32 && id_dtype != TT_I64) || !aligned_to(loss, 4)) return TT_EINVAL;
    if (tokens > 0 && (!aligned_to(actions, id_dtype == TT_I32 ? 4 : 8) || !aligned_to(old_logp, 4) || !aligned_to(advantage, 4) || !aligned_to(weight, 4) ||
                       (policy->kl != 0.0f && !aligned_to(ref_logp, 4)) || (logp && !aligned_to(logp, 4))))
        return TT_EINVAL;
    PolicyParams p;
    if (!make_blocks(X, tX, k, tokens, vocab, &p.X)) return TT_EINFEASIBLE;
    p.G = p.X;
    if (dX) {
        if (!make_blocks(const_cast<const void *const *>(dX), tdX, k, tokens, vocab, &p.G)) return TT_EINFEASIBLE;
    } else {
        for (void *&q : p.G.p) q = nullptr;
    }
    if (tokens > 0 && (!workspace || ws_bytes < policy_space(tokens) || reinterpret_cast<uintptr_t>(workspace) % 256)) return TT_EWORKSPACE;
    p.s = vocab > 0 ? pieces_of(p.X, p.G, vocab, 16 / e) : Pieces{1, 0, 0, 0};
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
    if (tokens > 0 && (st = launch_policy(p, dtype, id_dtype, s)) != TT_OK) return st;
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
    if (!(scale > 0.0f) || std::isinf(scale) || !shards_fit(X, k, e) || (id_dtype != TT_I32 && id_dtype != TT_I64)) return TT_EINVAL;
    if (tokens > 0 && (!aligned_to(ids, id_dtype == TT_I32 ? 4 : 8) || !aligned_to(logp, 4))) return TT_EINVAL;
    PolicyParams p;
    if (!make_blocks(X, tX, k, tokens, vocab, &p.X)) return TT_EINFEASIBLE;
    if (tokens == 0) return TT_OK;
    if (!workspace || ws_bytes < policy_space(tokens) || reinterpret_cast<uintptr_t>(workspace) % 256) return TT_EWORKSPACE;
    p.G = p.X;
    for (void *&q : p.G.p) q = nullptr;
    p.s = vocab > 0 ? pieces_of(p.X, p.G, vocab, 16 / e) : Pieces{1, 0, 0, 0};
    p.actions = ids;
    p.old_logp = p.ref_logp = p.advantage = p.weight = nullptr;
    p.logp = logp;
    p.row_loss = nullptr;
    p.tokens = (uint32_t)tokens;
    p.vocab = vocab;
    p.policy = tt_policy{scale, 0.0f, 0.0f, 0.0f};
    ProfileScope scope(stream, TT_K_LOSS, 1 << k, tokens, vocab, e, (uint64_t)tokens * (uint64_t)vocab * e, 0);
    return launch_policy(p, dtype, id_dtype, reinterpret_cast<hipStream_t>(stream));
}
