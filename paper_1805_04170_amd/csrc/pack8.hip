// Activations in 8 bits between a chain's forward and backward pass: blocks of 32 values of a row with a power of two each
// (tt_pack8, tt_unpack8), and a fully-connected layer's backward pass that reads them (tt_fc_backward_packed).
//
// Packing and unpacking are bound by memory: 3 bytes a bf16 value, and one byte per 32.  A power of two as the scale makes
// every step exact: value * 2^-e, its rounding, and q * 2^e in bf16's eight bits, so the backward products run on the
// 16-bit kernels and see exactly what the 8-bit form stands for.
#include <cstdint>
#include <cstring>
#include "launch_util.h"
#include "block_table.h"
#include "tensor_tiling_tokens.h"
#include "tt_wave.h"

namespace tt {
namespace {

constexpr int kThreads = 256, kBlock = TT_PACK8_BLOCK;

struct PackParams {
    void *X[kMaxShards];
    int8_t *Q[kMaxShards];
    uint8_t *S[kMaxShards];
    uint32_t rows, cols, bpr; // of a shard; blocks per row
    uint64_t units;           // half blocks per shard
};

// 2^-e of a block from the exponent byte e + 127, and the byte from the largest magnitude's bits
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    // 2^e >= top / 127, and 127 = 2^6 * 1.984375: one more where top's mantissa is above 1.984375's
    int e = (int)(top >> 23) - 127 - 6 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    if (e < -126) e = -126;
    return top >= 0x7f800000u ? 255u : (uint32_t)(e + 127);
}

// Two lanes a block, 16 values each (for the values a row does not have: zeros).
template <typename T> __global__ __launch_bounds__(kThreads) void pack8_kernel(const PackParams p)
{
    const uint64_t u = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    const bool on = u < p.units;
    const uint64_t blk = (on ? u : p.units - 1) >> 1;
    const uint32_t half = (uint32_t)u & 1u;
    const uint32_t row = (uint32_t)(blk / p.bpr), b = (uint32_t)(blk - (uint64_t)row * p.bpr);
    const uint32_t col = b * kBlock + half * 16;
    const uint32_t n = !on || col >= p.cols ? 0 : p.cols - col < 16 ? p.cols - col : 16;
    const size_t at = (size_t)row * p.cols + col;
    const T *x = static_cast<const T *>(p.X[blockIdx.y]) + at;
    float f[16];
    if (n == 16) {
        constexpr int EV = kVec<T>;
        u32x4 r[16 / EV];
#pragma unroll
        for (int i = 0; i < 16 / EV; ++i) r[i] = load16(x + i * EV);
#pragma unroll
        for (int i = 0; i < 16 / EV; ++i) {
            float g[EV];
            unpack16(r[i], g, T());
#pragma unroll
            for (int q = 0; q < EV; ++q) f[i * EV + q] = g[q];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = (uint32_t)i < n ? to_float(x[i]) : 0.0f;
    }
    uint32_t top = 0; // magnitudes compare as their bits do, infinities and NaN above all others
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t m = __float_as_uint(f[i]) & 0x7fffffffu;
        top = m > top ? m : top;
    }
    const uint32_t other = wave::shfl_xor(top, 1);
    top = other > top ? other : top;
    const uint32_t s = scale_byte(top);
    if (n == 0) return;
    const float inv = s == 255 ? 0.0f : __uint_as_float((254u - s) << 23);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        int q = s == 255 ? 0 : (int)rintf(f[i] * inv);
        if (q == 0 && s != 255) q = f[i] > 0.0f ? 1 : f[i] < 0.0f ? -1 : 0;
        w[i >> 2] |= (uint32_t)(q & 255) << (8 * (i & 3));
    }
    int8_t *to = p.Q[blockIdx.y] + at;
    if (n == 16) {
        typedef uint32_t any __attribute__((ext_vector_type(4), aligned(1)));
        *reinterpret_cast<any *>(to) = any{w[0], w[1], w[2], w[3]};
    } else {
        for (uint32_t i = 0; i < n; ++i) to[i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
    if (half == 0) p.S[blockIdx.y][blk] = (uint8_t)s;
}

__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s == 255 ? 0x7fc00000u : s << 23); }

// 16 values of a row from 8 bits (to: dense rows like Q's)
template <typename T> __device__ __forceinline__ void unpack_half_block(const PackParams &p, uint32_t shard, uint64_t u)
{
    const uint64_t blk = u >> 1;
    const uint32_t row = (uint32_t)(blk / p.bpr), b = (uint32_t)(blk - (uint64_t)row * p.bpr);
    const uint32_t col = b * kBlock + ((uint32_t)u & 1u) * 16;
    if (col >= p.cols) return;
    const uint32_t n = p.cols - col < 16 ? p.cols - col : 16;
    const size_t at = (size_t)row * p.cols + col;
    const int8_t *q = p.Q[shard] + at;
    T *x = static_cast<T *>(p.X[shard]) + at;
    const float s = scale_of(p.S[shard][blk]);
    if (n == 16) {
        typedef uint32_t any __attribute__((ext_vector_type(4), aligned(1)));
        const any w = *reinterpret_cast<const any *>(q);
        constexpr int EV = kVec<T>;
#pragma unroll
        for (int i = 0; i < 16 / EV; ++i) {
            float g[EV];
#pragma unroll
            for (int j = 0; j < EV; ++j) g[j] = (float)(int8_t)(w[(i * EV + j) >> 2] >> (8 * (j & 3))) * s;
            store16(x + i * EV, pack16(g, T()));
        }
    } else {
        for (uint32_t i = 0; i < n; ++i) x[i] = from_float<T>((float)q[i] * s);
    }
}

template <typename T> __global__ __launch_bounds__(kThreads) void unpack8_kernel(const PackParams p)
{
    const uint64_t u = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    if (u < p.units) unpack_half_block<T>(p, blockIdx.y, u);
}

// shard extents and the launch's size; `count` shards
tt_status pack_geometry(PackParams *p, int64_t srows, int64_t scols, dim3 *grid, int count)
{
    if (!fits31(srows) || !fits31(scols)) return TT_EUNSUPPORTED;
    p->rows = (uint32_t)srows;
    p->cols = (uint32_t)scols;
    p->bpr = (uint32_t)((scols + kBlock - 1) / kBlock);
    p->units = (uint64_t)srows * p->bpr * 2;
    const uint64_t g = (p->units + kThreads - 1) / kThreads;
    if (g * kThreads >= (uint64_t(1) << 32)) return TT_EUNSUPPORTED;
    *grid = dim3((uint32_t)g, (uint32_t)count);
    return TT_OK;
}

bool bytes_fit(const void *const *shards, int k)
{
    if (!shards) return false;
    for (int s = 0; s < (1 << k); ++s) if (!shards[s]) return false;
    return true;
}

tt_status launch_pack(bool pack, int64_t rows, int64_t cols, int k, int dtype, const tt_tiling &t, const void *const *X,
                      const void *const *Q, const void *const *S, void *stream)
{
    if (!valid_k(k) || !valid_tiling(t, k) || !valid_dtype(dtype) || rows < 0 || cols < 0) return TT_EINVAL;
    if (!shards_fit(X, k, dtype_bytes(dtype)) || !bytes_fit(Q, k) || !bytes_fit(S, k)) return TT_EINVAL;
    Grid g;
    if (!make_grid(t.cut, k, rows, cols, &g)) return TT_EINFEASIBLE;
    if (rows == 0 || cols == 0) return TT_OK;
    PackParams p;
    dim3 grid;
    const int n = 1 << k;
    const tt_status st = pack_geometry(&p, g.srows, g.scols, &grid, n);
    if (st != TT_OK) return st;
    for (int s = 0; s < kMaxShards; ++s) {
        p.X[s] = s < n ? const_cast<void *>(X[s]) : nullptr;
        p.Q[s] = s < n ? static_cast<int8_t *>(const_cast<void *>(Q[s])) : nullptr;
        p.S[s] = s < n ? static_cast<uint8_t *>(const_cast<void *>(S[s])) : nullptr;
    }
    const uint64_t values = (uint64_t)g.srows * g.scols * n;
    ProfileScope scope(stream, pack ? TT_K_PACK : TT_K_UNPACK, n, rows, cols, dtype_bytes(dtype), values * (dtype_bytes(dtype) + 1) + (uint64_t)g.srows * p.bpr * n, 0);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (pack) {
        if (dtype == TT_BF16) hipLaunchKernelGGL((pack8_kernel<uint16_t>), grid, dim3(kThreads), 0, s, p);
        else hipLaunchKernelGGL((pack8_kernel<float>), grid, dim3(kThreads), 0, s, p);
    } else {
        if (dtype == TT_BF16) hipLaunchKernelGGL((unpack8_kernel<uint16_t>), grid, dim3(kThreads), 0, s, p);
        else hipLaunchKernelGGL((unpack8_kernel<float>), grid, dim3(kThreads), 0, s, p);
    }
    return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
}

template <typename P> const void *const *untyped(P *const *p) { return reinterpret_cast<const void *const *>(p); }

// The workspace of a backward pass from 8 bits: the activations unpacked, one buffer per shard of X and of Y, then what the
// 16-bit pass asks for.
struct PackedSpace {
    Grid x, y;
    size_t x_pitch = 0, y_pitch = 0, inner_at = 0, bytes = 0;
};

tt_status packed_space(const tt_layer *layer, int64_t batch, int k, int dtype, const tt_tiling &tX, const tt_tiling &tW, const tt_tiling &tY,
                       const tt_tiling &tdY, const tt_tiling &tdX, const uint8_t *fd, const uint8_t *fw, int with_dx, PackedSpace *s)
{
    size_t inner = 0;
    const tt_status st = tt_fc_workspace_bytes(layer, batch, k, dtype, TT_OP_DGRAD, tX, tW, tY, tdY, tdX, fd, fw, with_dx, &inner);
    if (st != TT_OK) return st; // (checks the layer, the types and the tilings)
    if (!make_grid(tX.cut, k, batch, layer->n_in, &s->x)) return TT_EINFEASIBLE;
    const size_t e = (size_t)dtype_bytes(dtype);
    s->x_pitch = align_up((size_t)s->x.srows * s->x.scols * e, 256);
    if (layer->act == TT_ACT_RELU) {
        if (!make_grid(tY.cut, k, batch, layer->n_out, &s->y)) return TT_EINFEASIBLE;
        s->y_pitch = align_up((size_t)s->y.srows * s->y.scols * e, 256);
    }
    s->inner_at = (s->x_pitch + s->y_pitch) << k;
    s->bytes = s->inner_at + inner;
    return TT_OK;
}

} // namespace
} // namespace tt

extern "C" tt_status tt_pack8(int64_t rows, int64_t cols, int k, int dtype, tt_tiling t, const void *const *X, int8_t *const *Q,
                              uint8_t *const *S, void *stream)
{
    return tt::launch_pack(true, rows, cols, k, dtype, t, X, tt::untyped(Q), tt::untyped(S), stream);
}

extern "C" tt_status tt_unpack8(int64_t rows, int64_t cols, int k, int dtype, tt_tiling t, const int8_t *const *Q, const uint8_t *const *S,
                                void *const *X, void *stream)
{
    return tt::launch_pack(false, rows, cols, k, dtype, t, tt::untyped(X), tt::untyped(Q), tt::untyped(S), stream);
}

extern "C" tt_status tt_fc_packed_workspace_bytes(const tt_layer *layer, int64_t batch, int k, int dtype, tt_tiling tX, tt_tiling tW,
                                                  tt_tiling tY, tt_tiling tdY, tt_tiling tdX, const uint8_t *forms_dgrad,
                                                  const uint8_t *forms_wgrad, int with_dx, size_t *bytes)
{
    if (!bytes) return TT_EINVAL;
    tt::PackedSpace s;
    const tt_status st = tt::packed_space(layer, batch, k, dtype, tX, tW, tY, tdY, tdX, forms_dgrad, forms_wgrad, with_dx, &s);
    if (st != TT_OK) return st;
    *bytes = s.bytes;
    return TT_OK;
}

extern "C" tt_status tt_fc_backward_packed(const tt_layer *layer, int64_t batch, int k, int dtype, tt_tiling tX, tt_tiling tW,
                                           tt_tiling tY, tt_tiling tdY, tt_tiling tdX, const uint8_t *forms_dgrad,
                                           const uint8_t *forms_wgrad, const int8_t *const *XQ, const uint8_t *const *XS,
                                           const void *const *W, const int8_t *const *YQ, const uint8_t *const *YS,
                                           const void *const *dY, void *const *dX, void *const *dW, void *workspace, size_t ws_bytes,
                                           void *stream)
{
    using namespace tt;
    PackedSpace s;
    tt_status st = packed_space(layer, batch, k, dtype, tX, tW, tY, tdY, tdX, forms_dgrad, forms_wgrad, dX != nullptr, &s);
    if (st != TT_OK) return st;
    const int e = dtype_bytes(dtype);
    const bool relu = layer->act == TT_ACT_RELU;
    // everything is checked before the first launch
    if (!bytes_fit(untyped(XQ), k) || !bytes_fit(untyped(XS), k) || (relu && (!bytes_fit(untyped(YQ), k) || !bytes_fit(untyped(YS), k)))) return TT_EINVAL;
    if (!shards_fit(W, k, e) || !shards_fit(dY, k, e) || !shards_fit(const_cast<const void *const *>(dW), k, e) ||
        (dX && !shards_fit(const_cast<const void *const *>(dX), k, e)))
        return TT_EINVAL;
    if (!workspace || ws_bytes < s.bytes || reinterpret_cast<uintptr_t>(workspace) % 256) return TT_EWORKSPACE;
    char *ws = static_cast<char *>(workspace);
    void *X[kMaxShards], *Y[kMaxShards];
    for (int i = 0; i < (1 << k); ++i) {
        X[i] = ws + (size_t)i * s.x_pitch;
        Y[i] = ws + (s.x_pitch << k) + (size_t)i * s.y_pitch;
    }
    if ((st = launch_pack(false, batch, layer->n_in, k, dtype, tX, X, untyped(XQ), untyped(XS), stream)) != TT_OK) return st;
    if (relu && (st = launch_pack(false, batch, layer->n_out, k, dtype, tY, Y, untyped(YQ), untyped(YS), stream)) != TT_OK) return st;
    return tt_fc_backward(layer, batch, k, dtype, tX, tW, tY, tdY, tdX, forms_dgrad, forms_wgrad, X, W, relu ? Y : nullptr, dY, dX, dW,
                          ws + s.inner_at, ws_bytes - s.inner_at, stream);
}
