// Activations in 8 bits between a chain's forward and backward pass: blocks of 32 values of a row with a power of two each
// (tt_pack8, tt_unpack8), and a fully-connected layer's backward pass that reads them (tt_fc_backward_packed).
//
// Packing and unpacking are bound by memory: 3 bytes a bf16 value, and one byte per 32.  A power of two as the scale makes
// every step exact: value * 2^-e, its rounding, and q * 2^e in bf16's eight bits, so the backward products run on the
// 16-bit kernels and see exactly what the 8-bit form stands for.  8192 x 8192 bf16 values: packed in 46 us, unpacked in 32, 5.2 TB/s
// together (an elementwise pass over as many bytes reaches 5.8); 8192 x 4096 fp32 values 40 and 44, 4.0.
#include <cstdint>
#include <cstring>
#include "launch_util.h"
#include "tiled_rows.h"

namespace tt {
namespace {

constexpr int kThreads = 256, kBlock = TT_PACK8_BLOCK;

struct PackParams {
    void *X[kMaxShards];
    int8_t *Q[kMaxShards];
    uint8_t *S[kMaxShards];
    uint32_t cols;   // of a shard
    Divisor by_bpr;  // blocks per row
    uint32_t narrow; // blocks are counted in 31 bits
    uint64_t units;  // half blocks per shard
};

// 2^-e of a block from the exponent byte e + 127, and the byte from the largest magnitude's bits
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    // 2^e >= top / 127, and 127 = 2^6 * 1.984375: one more where top's mantissa is above 1.984375's
    int e = (int)(top >> 23) - 127 - 6 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    if (e < -126) e = -126;
    return top >= 0x7f800000u ? 255u : (uint32_t)(e + 127);
}

// Where half a block lies: 16 values of a row (n of them are there)
struct Half { uint64_t block; size_t at; uint32_t n; };
__device__ __forceinline__ Half half_of(const PackParams &p, uint64_t u)
{
    const uint64_t blk = u >> 1;
    const uint32_t row = p.narrow ? quotient((uint32_t)blk, p.by_bpr) : (uint32_t)(blk / p.by_bpr.d), b = (uint32_t)(blk - (uint64_t)row * p.by_bpr.d);
    const uint32_t col = b * kBlock + ((uint32_t)u & 1u) * 16;
    return {blk, (size_t)row * p.cols + col, u >= p.units || col >= p.cols ? 0 : p.cols - col < 16 ? p.cols - col : 16};
}
template <typename T> struct Values { u32x4 r[16 / kVec<T>]; };
template <typename T> __device__ __forceinline__ Values<T> load_values(const T *x, uint32_t n)
{
    Values<T> v;
#pragma unroll
    for (int i = 0; i < 16 / kVec<T>; ++i) {
        const uint32_t left = n > (uint32_t)(i * kVec<T>) ? n - i * kVec<T> : 0;
        v.r[i] = left >= (uint32_t)kVec<T> ? load16(x + i * kVec<T>) : load_part(x + i * kVec<T>, left);
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store_values(T *x, const Values<T> &v, uint32_t n)
{
#pragma unroll
    for (int i = 0; i < 16 / kVec<T>; ++i) {
        const uint32_t left = n > (uint32_t)(i * kVec<T>) ? n - i * kVec<T> : 0;
        if (left >= (uint32_t)kVec<T>) store16(x + i * kVec<T>, v.r[i]);
        else store_part(x + i * kVec<T>, v.r[i], left);
    }
}
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
__device__ __forceinline__ u32x4 load_bytes(const int8_t *q, uint32_t n)
{
    if (n == 16) {
        const u32x4_any w = *(const TT_GLOBAL u32x4_any *)q;
        return u32x4{w.x, w.y, w.z, w.w};
    }
    uint32_t w[4] = {0, 0, 0, 0};
    for (uint32_t i = 0; i < n; ++i) w[i >> 2] |= (uint32_t)(uint8_t)load1(q + i) << (8 * (i & 3));
    return u32x4{w[0], w[1], w[2], w[3]};
}

// The largest magnitude's bits of a vector: magnitudes compare as their bits do, infinities and NaN above all others
__device__ __forceinline__ uint32_t largest(u32x4 v, float)
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t m = v[j] & 0x7fffffffu;
        top = m > top ? m : top;
    }
    return top;
}
__device__ __forceinline__ uint32_t largest(u32x4 v, uint16_t)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t m = v[j] & 0x7fff7fffu;
        top = __builtin_elementwise_max(top, u16x2{(uint16_t)m, (uint16_t)(m >> 16)});
    }
    return (uint32_t)(top.x > top.y ? top.x : top.y) << 16;
}
// x / step in whole steps (low byte), ties to even, a step at least where x is not 0 (a magnitude of 0.75 rounds to one): x inv is exact,
// and 1.5 * 2^23 + n is n in the number's last bits.  Comparisons would cost more: each waits for its result.
__device__ __forceinline__ uint32_t steps_of(float x, float inv)
{
    const float least = fminf(fabsf(ldexpf(x, 160)), 0.75f); // 0 for 0, 0.75 for anything else, the smallest denormal too
    return __float_as_uint(copysignf(fmaxf(fabsf(x * inv), least), x) + 12582912.0f);
}

__device__ __forceinline__ float inverse_of(uint32_t s) { return s == 255 ? 0.0f : __uint_as_float((254u - s) << 23); }
// a vector's values as bytes
template <typename T> struct Bytes { uint32_t w[kVec<T> / 4]; };
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));
__device__ __forceinline__ void load_bytes(const int8_t *q, Bytes<uint16_t> &b)
{
    const u32x2_any w = *(const TT_GLOBAL u32x2_any *)q;
    b.w[0] = w.x;
    b.w[1] = w.y;
}
__device__ __forceinline__ void load_bytes(const int8_t *q, Bytes<float> &b) { b.w[0] = *(const TT_GLOBAL u32_any *)q; }
template <typename T> __device__ __forceinline__ Bytes<T> packed(u32x4 v, uint32_t s)
{
    const float inv = inverse_of(s);
    float g[kVec<T>];
    unpack16(v, g, T());
    Bytes<T> b;
#pragma unroll
    for (int i = 0; i < kVec<T> / 4; ++i) {
        b.w[i] = wave::low_bytes(steps_of(g[4 * i], inv), steps_of(g[4 * i + 1], inv), steps_of(g[4 * i + 2], inv), steps_of(g[4 * i + 3], inv));
        if (s == 255) b.w[i] = 0;
    }
    return b;
}

// Any width: two lanes a block, 16 values each.
template <typename T> __global__ __launch_bounds__(kThreads) void pack8_kernel(const PackParams p)
{
    const uint64_t u = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    const Half h = half_of(p, u);
    const Values<T> v = load_values(static_cast<const T *>(p.X[blockIdx.y]) + (h.n ? h.at : 0), h.n);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16 / kVec<T>; ++i) {
        const uint32_t t = largest(v.r[i], T());
        top = t > top ? t : top;
    }
    const uint32_t other = wave::shfl_xor(top, 1), s = scale_byte(other > top ? other : top);
    if (h.n == 0) return;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 16 / kVec<T>; ++i) {
        const Bytes<T> b = packed<T>(v.r[i], s);
#pragma unroll
        for (int j = 0; j < kVec<T> / 4; ++j) w[i * kVec<T> / 4 + j] = b.w[j];
    }
    int8_t *to = p.Q[blockIdx.y] + h.at;
    if (h.n == 16) {
        *(TT_GLOBAL u32x4_any *)to = u32x4_any{w[0], w[1], w[2], w[3]};
    } else {
        for (uint32_t i = 0; i < h.n; ++i) store1(to + i, (int8_t)(w[i >> 2] >> (8 * (i & 3))));
    }
    if ((threadIdx.x & 1u) == 0) store1(p.S[blockIdx.y] + h.block, (uint8_t)s);
}

// 2^(s - 127), NaN for 255.  (s = 0, which packing never makes, is a denormal; steps of it are exact in bf16 as well.)
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s == 255 ? 0x7fc00000u : s == 0 ? 0x00400000u : s << 23); }
// byte i of a vector, signed
__device__ __forceinline__ int byte_of(const u32x4 &w, int i) { return (int)(int8_t)(w[i >> 2] >> (8 * (i & 3))); }

// 16 values of a row from 8 bits
template <typename T> __device__ __forceinline__ Values<T> values_from(u32x4 q, float scale)
{
    Values<T> v;
#pragma unroll
    for (int i = 0; i < 16 / kVec<T>; ++i) {
        float g[kVec<T>];
#pragma unroll
        for (int j = 0; j < kVec<T>; ++j) g[j] = (float)byte_of(q, i * kVec<T> + j) * scale;
        v.r[i] = pack16(g, T());
    }
    return v;
}

template <typename T> __device__ __forceinline__ void unpack_half_block(const PackParams &p, uint32_t shard, uint64_t u)
{
    const Half h = half_of(p, u);
    if (h.n == 0) return;
    const u32x4 q = load_bytes(p.Q[shard] + h.at, h.n);
    store_values(static_cast<T *>(p.X[shard]) + h.at, values_from<T>(q, scale_of(load1(p.S[shard] + h.block))), h.n);
}

template <typename T> __global__ __launch_bounds__(kThreads) void unpack8_kernel(const PackParams p)
{
    const uint64_t u = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    unpack_half_block<T>(p, blockIdx.y, u);
}

// Rows of whole blocks: a shard is one row of blocks.  A lane takes a vector, 4 (bf16) or 8 lanes a block, so that a wave's loads and
// stores are one piece of memory each, and kFlat vectors are on their way together.  GATE: what is written is dY where the value is
// above 0.
constexpr int kFlat = 4;
template <typename T, bool GATE> __device__ __forceinline__ void unpack_flat(const PackParams &p, uint32_t shard, uint32_t group, const T *dY)
{
    constexpr uint32_t EV = kVec<T>, LANES = kBlock / EV;
    const uint64_t j0 = (uint64_t)group * (kThreads * kFlat) + threadIdx.x, last = p.units * (16 / EV) - 1;
    Bytes<T> q[kFlat];
    uint32_t s[kFlat];
    u32x4 v[kFlat];
#pragma unroll
    for (int k = 0; k < kFlat; ++k) {
        const uint64_t j = j0 + k * kThreads < last ? j0 + k * kThreads : last;
        load_bytes(p.Q[shard] + j * EV, q[k]);
        s[k] = load1(p.S[shard] + j / LANES);
        if constexpr (GATE) v[k] = load16(dY + j * EV);
    }
#pragma unroll
    for (int k = 0; k < kFlat; ++k) {
        const uint64_t j = j0 + k * kThreads;
        if (j > last) continue;
        if constexpr (GATE) {
#pragma unroll
            for (uint32_t i = 0; i < EV; ++i) {
                const bool open = s[k] != 255 && (int8_t)(q[k].w[i / 4] >> (8 * (i & 3))) > 0;
                const uint32_t mine = sizeof(T) == 4 ? 0xffffffffu : i & 1 ? 0xffff0000u : 0x0000ffffu;
                v[k][i * sizeof(T) / 4] &= open ? 0xffffffffu : ~mine;
            }
        } else {
            const float scale = scale_of(s[k]);
            float g[EV];
#pragma unroll
            for (uint32_t i = 0; i < EV; ++i) g[i] = (float)(int8_t)(q[k].w[i / 4] >> (8 * (i & 3))) * scale;
            v[k] = pack16(g, T());
        }
        store16(static_cast<T *>(p.X[shard]) + j * EV, v[k]);
    }
}
// What a layer's backward pass needs of its activations, in one launch: the input unpacked, and the output's gradient where the
// output's value is above 0 (the output itself is read as its 8 bits and never written out).
struct GateParams {
    PackParams x;          // blocks of the input: Q, S, X written
    const void *dY[kMaxShards];
    PackParams y;          // blocks of the output: Q, S; X takes the gated gradient
    uint32_t x_blocks;
};
// (both of whole blocks)
template <typename T> __global__ __launch_bounds__(kThreads) void unpack_gate_flat_kernel(const GateParams p)
{
    if (blockIdx.y < p.x_blocks) unpack_flat<T, false>(p.x, blockIdx.y, blockIdx.x, nullptr);
    else unpack_flat<T, true>(p.y, blockIdx.y - p.x_blocks, blockIdx.x, static_cast<const T *>(p.dY[blockIdx.y - p.x_blocks]));
}
template <typename T> __global__ __launch_bounds__(kThreads) void unpack_gate_kernel(const GateParams p)
{
    const uint64_t u = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    if (blockIdx.y < p.x_blocks) {
        unpack_half_block<T>(p.x, blockIdx.y, u);
        return;
    }
    const uint32_t b = blockIdx.y - p.x_blocks;
    const Half h = half_of(p.y, u);
    if (h.n == 0) return;
    Values<T> v = load_values(static_cast<const T *>(p.dY[b]) + h.at, h.n);
    const u32x4 q = load_bytes(p.y.Q[b] + h.at, h.n);
    const bool number = load1(p.y.S[b] + h.block) != 255;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const bool open = number && byte_of(q, i) > 0;
        const uint32_t mine = sizeof(T) == 4 ? 0xffffffffu : i & 1 ? 0xffff0000u : 0x0000ffffu;
        v.r[i / kVec<T>][i % kVec<T> * (int)sizeof(T) / 4] &= open ? 0xffffffffu : ~mine;
    }
    store_values(static_cast<T *>(p.y.X[b]) + h.at, v, h.n);
}

bool flat(const PackParams &p) { return p.cols % kBlock == 0; }
// workgroups for a shard: 16 values a lane, or kFlat vectors
uint64_t groups_of(const PackParams &p) { return (p.units + kThreads - 1) / kThreads; }
uint64_t flat_groups_of(const PackParams &p, int elem_bytes) { return (p.units * elem_bytes + kThreads * kFlat - 1) / (kThreads * kFlat); }
tt_status pack_geometry(PackParams *p, int64_t srows, int64_t scols)
{
    if (!fits31(srows) || !fits31(scols)) return TT_EUNSUPPORTED;
    p->cols = (uint32_t)scols;
    const uint32_t bpr = (uint32_t)((scols + kBlock - 1) / kBlock);
    p->by_bpr = divisor(bpr);
    p->units = (uint64_t)srows * bpr * 2;
    p->narrow = p->units / 2 + kThreads < (uint64_t(1) << 31);
    return p->units >= (uint64_t(1) << 32) - kThreads ? TT_EUNSUPPORTED : TT_OK; // (a launch holds fewer than 2^32 threads)
}
template <typename T> void launch_unpack(const PackParams &p, int count, hipStream_t s)
{
    hipLaunchKernelGGL((unpack8_kernel<T>), dim3((uint32_t)groups_of(p), (uint32_t)count), dim3(kThreads), 0, s, p);
}
template <typename T> void launch_pack(const PackParams &p, int count, hipStream_t s)
{
    hipLaunchKernelGGL((pack8_kernel<T>), dim3((uint32_t)groups_of(p), (uint32_t)count), dim3(kThreads), 0, s, p);
}
// Pieces of memory where both tensors have them (2048 x 8192 twice: 24 us, 5.5 TB/s, against 29 by halves of blocks; packing and
// unpacking by themselves are as fast either way).
template <typename T> void launch_unpack_gate(const GateParams &p, uint32_t y_blocks, hipStream_t s)
{
    const bool both = flat(p.x) && flat(p.y);
    const uint64_t x = both ? flat_groups_of(p.x, (int)sizeof(T)) : groups_of(p.x), y = both ? flat_groups_of(p.y, (int)sizeof(T)) : groups_of(p.y);
    const dim3 grid((uint32_t)(x > y ? x : y), p.x_blocks + y_blocks);
    if (both) hipLaunchKernelGGL((unpack_gate_flat_kernel<T>), grid, dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((unpack_gate_kernel<T>), grid, dim3(kThreads), 0, s, p);
}

bool bytes_fit(const void *const *shards, int k, bool empty = false)
{
    if (!shards || empty) return shards != nullptr;
    for (int s = 0; s < (1 << k); ++s) if (!shards[s]) return false;
    return true;
}

tt_status run_pack(bool pack, int64_t rows, int64_t cols, int k, int dtype, const tt_tiling &t, const void *const *X,
                      const void *const *Q, const void *const *S, void *stream)
{
    if (!valid_k(k) || !valid_tiling(t, k) || !valid_dtype(dtype) || rows < 0 || cols < 0) return TT_EINVAL;
    const bool empty = rows == 0 || cols == 0;
    if (!shards_fit(X, k, dtype_bytes(dtype), empty) || !bytes_fit(Q, k, empty) || !bytes_fit(S, k, empty)) return TT_EINVAL;
    Grid g;
    if (!make_grid(t.cut, k, rows, cols, &g)) return TT_EINFEASIBLE;
    if (empty) return TT_OK;
    PackParams p;
    const int n = 1 << k;
    const tt_status st = pack_geometry(&p, g.srows, g.scols);
    if (st != TT_OK) return st;
    for (int s = 0; s < kMaxShards; ++s) {
        p.X[s] = s < n ? const_cast<void *>(X[s]) : nullptr;
        p.Q[s] = s < n ? static_cast<int8_t *>(const_cast<void *>(Q[s])) : nullptr;
        p.S[s] = s < n ? static_cast<uint8_t *>(const_cast<void *>(S[s])) : nullptr;
    }
    const uint64_t values = (uint64_t)g.srows * g.scols * n;
    ProfileScope scope(stream, pack ? TT_K_PACK : TT_K_UNPACK, n, rows, cols, dtype_bytes(dtype), values * (dtype_bytes(dtype) + 1) + (uint64_t)g.srows * p.by_bpr.d * n, 0);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (pack) {
        if (dtype == TT_BF16) launch_pack<uint16_t>(p, n, s);
        else launch_pack<float>(p, n, s);
    } else {
        if (dtype == TT_BF16) launch_unpack<uint16_t>(p, n, s);
        else launch_unpack<float>(p, n, s);
    }
    return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
}

template <typename P> const void *const *untyped(P *const *p) { return reinterpret_cast<const void *const *>(p); }

// The workspace of a backward pass from 8 bits: the input's blocks unpacked; where the output and its gradient are cut into blocks
// alike, the gated gradient's blocks, otherwise the output's unpacked; then what the 16-bit pass asks for.  Replicas share a
// block's buffer: that pass only reads them.
struct PackedSpace {
    BlockTable x, y, dy;
    bool relu = false, gated = false;
    tt_layer layer; // of the 16-bit pass
    size_t x_pitch = 0, y_pitch = 0, y_at = 0, inner_at = 0, bytes = 0;
};
uint32_t blocks_of(const BlockTable &b) { return b.nR * b.nC; }

tt_status packed_space(const tt_layer *layer, int64_t batch, int k, int dtype, const tt_tiling &tX, const tt_tiling &tW, const tt_tiling &tY,
                       const tt_tiling &tdY, const tt_tiling &tdX, const uint8_t *fd, const uint8_t *fw, int with_dx, PackedSpace *s)
{
    size_t inner = 0;
    tt_status st = tt_fc_workspace_bytes(layer, batch, k, dtype, TT_OP_DGRAD, tX, tW, tY, tdY, tdX, fd, fw, with_dx, &inner);
    if (st != TT_OK) return st; // (checks the layer, the types and the tilings)
    if (!fits31(batch) || !fits31(layer->n_in) || !fits31(layer->n_out)) return TT_EUNSUPPORTED;
    s->layer = *layer;
    s->relu = layer->act == TT_ACT_RELU;
    if (!make_blocks(nullptr, tX, k, batch, layer->n_in, &s->x) || !make_blocks(nullptr, tdY, k, batch, layer->n_out, &s->dy)) return TT_EINFEASIBLE;
    const size_t e = (size_t)dtype_bytes(dtype);
    s->x_pitch = align_up((size_t)s->x.srows * s->x.scols * e, 256);
    s->y_at = s->inner_at = s->x_pitch * blocks_of(s->x);
    if (s->relu) {
        if (!make_blocks(nullptr, tY, k, batch, layer->n_out, &s->y)) return TT_EINFEASIBLE;
        s->gated = s->y.nR == s->dy.nR && s->y.nC == s->dy.nC;
        s->y_pitch = align_up((size_t)s->y.srows * s->y.scols * e, 256);
        s->inner_at += s->y_pitch * blocks_of(s->y);
    }
    if (s->gated) {
        s->layer.act = TT_ACT_NONE;
        st = tt_fc_workspace_bytes(&s->layer, batch, k, dtype, TT_OP_DGRAD, tX, tW, tY, tdY, tdX, fd, fw, with_dx, &inner);
        if (st != TT_OK) return st;
    }
    s->bytes = s->inner_at + inner;
    return TT_OK;
}

// one buffer per block: the block a shard holds
void buffers_of(void **shards, const tt_tiling &t, int k, const BlockTable &b, char *base, size_t pitch)
{
    Grid g;
    if (!make_grid(t.cut, k, (int64_t)b.srows * b.nR, (int64_t)b.scols * b.nC, &g)) return;
    for (uint32_t s = 0; s < (1u << k); ++s) shards[s] = base + (size_t)(extract(s, g.maskR, k) * b.nC + extract(s, g.maskC, k)) * pitch;
}

// the blocks of a tensor in 8 bits, one replica of each, and where their values go
tt_status packed_blocks(PackParams *p, const tt_tiling &t, int k, int64_t rows, int64_t cols, const void *const *Q, const void *const *S, char *to,
                        size_t pitch)
{
    BlockTable q, s;
    if (!make_blocks(Q, t, k, rows, cols, &q) || !make_blocks(S, t, k, rows, cols, &s)) return TT_EINFEASIBLE;
    const uint32_t n = blocks_of(q);
    for (uint32_t b = 0; b < (uint32_t)kMaxShards; ++b) {
        p->X[b] = b < n ? to + b * pitch : nullptr;
        p->Q[b] = b < n ? static_cast<int8_t *>(q.p[b * q.nrep]) : nullptr;
        p->S[b] = b < n ? static_cast<uint8_t *>(s.p[b * s.nrep]) : nullptr;
    }
    return pack_geometry(p, q.srows, q.scols);
}

} // namespace
} // namespace tt

extern "C" tt_status tt_pack8(int64_t rows, int64_t cols, int k, int dtype, tt_tiling t, const void *const *X, int8_t *const *Q,
                              uint8_t *const *S, void *stream)
{
    return tt::run_pack(true, rows, cols, k, dtype, t, X, tt::untyped(Q), tt::untyped(S), stream);
}

extern "C" tt_status tt_unpack8(int64_t rows, int64_t cols, int k, int dtype, tt_tiling t, const int8_t *const *Q, const uint8_t *const *S,
                                void *const *X, void *stream)
{
    return tt::run_pack(false, rows, cols, k, dtype, t, tt::untyped(X), tt::untyped(Q), tt::untyped(S), stream);
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
    buffers_of(X, tX, k, s.x, ws, s.x_pitch);
    GateParams p;
    if ((st = packed_blocks(&p.x, tX, k, batch, layer->n_in, untyped(XQ), untyped(XS), ws, s.x_pitch)) != TT_OK) return st;
    if (s.relu) {
        if ((st = packed_blocks(&p.y, tY, k, batch, layer->n_out, untyped(YQ), untyped(YS), ws + s.y_at, s.y_pitch)) != TT_OK) return st;
        buffers_of(Y, s.gated ? tdY : tY, k, s.gated ? s.dy : s.y, ws + s.y_at, s.y_pitch);
    }
    const hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
    const bool bf16 = dtype == TT_BF16;
    const uint64_t nx = (uint64_t)batch * layer->n_in, ny = (uint64_t)batch * layer->n_out;
    p.x_blocks = blocks_of(s.x);
    if (s.gated) {
        BlockTable dy;
        if (!make_blocks(dY, tdY, k, batch, layer->n_out, &dy)) return TT_EINFEASIBLE;
        const uint32_t n = blocks_of(dy);
        for (uint32_t b = 0; b < (uint32_t)kMaxShards; ++b) p.dY[b] = b < n ? dy.p[b * dy.nrep] : nullptr;
        ProfileScope scope(stream, TT_K_UNPACK, 1 << k, batch, layer->n_in + layer->n_out, e, nx * (e + 1) + ny * (2 * e + 1), 0);
        if (bf16) launch_unpack_gate<uint16_t>(p, n, hs);
        else launch_unpack_gate<float>(p, n, hs);
    } else {
        ProfileScope scope(stream, TT_K_UNPACK, 1 << k, batch, layer->n_in, e, nx * (e + 1), 0);
        if (bf16) launch_unpack<uint16_t>(p.x, (int)p.x_blocks, hs);
        else launch_unpack<float>(p.x, (int)p.x_blocks, hs);
    }
    if (s.relu && !s.gated) {
        ProfileScope scope(stream, TT_K_UNPACK, 1 << k, batch, layer->n_out, e, ny * (e + 1), 0);
        if (bf16) launch_unpack<uint16_t>(p.y, (int)blocks_of(s.y), hs);
        else launch_unpack<float>(p.y, (int)blocks_of(s.y), hs);
    }
    if (hipGetLastError() != hipSuccess) return TT_EDEVICE;
    return tt_fc_backward(&s.layer, batch, k, dtype, tX, tW, tY, tdY, tdX, forms_dgrad, forms_wgrad, X, W, s.gated ? nullptr : s.relu ? Y : nullptr,
                          s.gated ? Y : dY, dX, dW, ws + s.inner_at, ws_bytes - s.inner_at, stream);
}
