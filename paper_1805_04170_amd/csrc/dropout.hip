// Dropout (tt_dropout): which values are dropped is worked out from their place, nothing but the values is read and written.
//
// Bound by memory, with the generator beside it (ten rounds of two 32 x 32 bit products for a vector of 8 values).  16384 x 4096 bf16
// 47.6 us, 5.6 TB/s (an elementwise pass over as much reaches 5.95); 8192 x 4096 fp32 47.7.
#include <cstdint>
#include "launch_util.h"
#include "philox.h"
#include "row_reduce.h"

namespace tt {
namespace {

constexpr int kThreads = 256, kVectors = 4; // of a thread

struct DropoutParams {
    BlockTable X, Y;
    RowShape r;
    DropParams d;
    uint64_t units;   // vectors of the tensor
    uint32_t small;   // they are counted in 31 bits
    uint32_t once;    // results are stored past the caches
    Divisor by_units; // vectors of a row
};

template <typename T, bool CUT, bool NARROW> __global__ __launch_bounds__(kThreads) void dropout_kernel(const DropoutParams p)
{
    constexpr uint32_t EV = kVec<T>;
    const DropState d = drop_state(p.d);
    // the workgroup's first vector, and every lane's from there
    const uint64_t first = (uint64_t)blockIdx.x * (kThreads * kVectors);
    const uint32_t row0 = p.small ? quotient((uint32_t)first, p.by_units) : uniform((uint32_t)(first / p.r.units)), j0 = (uint32_t)(first - (uint64_t)row0 * p.r.units);
    const uint64_t left = p.units - first;
    uint32_t row[kVectors];
    Spot v[kVectors];
    u32x4 x[kVectors];
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        const uint32_t u = threadIdx.x + i * kThreads, j = j0 + (u < left ? u : 0); // (past the end: the workgroup's first vector again)
        const uint32_t over = quotient(j, p.by_units);
        row[i] = row0 + over;
        v[i] = spot_of<EV>(p.r, j - over * p.r.units);
        x[i] = load_spot<T, NARROW>(p.X, lane_of<CUT>(p.X, p.r.s, p.r.s.a_shift, row[i], v[i]), v[i]);
    }
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        float f[EV];
        unpack16(x[i], f, T());
        drop_values(d, row[i], v[i].q * p.r.s.seg + v[i].at, f);
        store_spot<T, CUT, NARROW>(p.Y, lane_of<CUT>(p.Y, p.r.s, p.r.s.b_shift, row[i], v[i]), v[i], pack16(f, T()), p.once);
    }
}

template <typename T> void launch_dropout(const DropoutParams &p, hipStream_t s)
{
    const dim3 grid((uint32_t)((p.units + kThreads * kVectors - 1) / (kThreads * kVectors))), block(kThreads);
    if (narrow_segments(p.r, kVec<T>)) hipLaunchKernelGGL((dropout_kernel<T, true, true>), grid, block, 0, s, p);
    else if (uncut(p.X) && uncut(p.Y)) hipLaunchKernelGGL((dropout_kernel<T, false, false>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((dropout_kernel<T, true, false>), grid, block, 0, s, p);
}

} // namespace
} // namespace tt

extern "C" tt_status tt_dropout(const tt_drop *drop, int64_t rows, int64_t cols, int k, int dtype, tt_tiling tX, tt_tiling tY,
                                const void *const *X, void *const *Y, void *stream)
{
    using namespace tt;
    DropoutParams p;
    if (!drop || !make_drop(drop, &p.d)) return TT_EINVAL;
    if (!valid_k(k) || !valid_tiling(tX, k) || !valid_tiling(tY, k) || !valid_dtype(dtype) || rows < 0 || cols < 0) return TT_EINVAL;
    const bool empty = rows == 0 || cols == 0;
    const int e = dtype_bytes(dtype);
    if (!shards_fit(X, k, e, empty) || !shards_fit(const_cast<const void *const *>(Y), k, e, empty)) return TT_EINVAL;
    if (!fits31(rows) || !fits31(cols)) return TT_EUNSUPPORTED;
    if (!make_blocks(X, tX, k, rows, cols, &p.X) || !make_blocks(const_cast<const void *const *>(Y), tY, k, rows, cols, &p.Y)) return TT_EINFEASIBLE;
    if (empty) return TT_OK;
    p.r = row_shape(p.X, p.Y, cols, 16 / e);
    p.by_units = divisor(p.r.units);
    p.units = (uint64_t)rows * p.r.units;
    p.small = p.units < (uint64_t(1) << 31);
    p.once = (uint64_t)rows * cols * e * p.Y.nrep >= kOnceBytes;
    if ((uint64_t)rows * (uint64_t)cols >= (uint64_t(1) << 37) || p.units / kVectors >= (uint64_t(1) << 32) - kThreads || p.r.units >= (1u << 31) - kThreads * kVectors)
        return TT_EUNSUPPORTED; // (a launch holds fewer than 2^32 threads)
    ProfileScope scope(stream, TT_K_DROPOUT, 1 << k, rows, cols, e, (uint64_t)rows * cols * e * (1 + p.Y.nrep), 0);
    if (dtype == TT_BF16) launch_dropout<uint16_t>(p, static_cast<hipStream_t>(stream));
    else launch_dropout<float>(p, static_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? TT_OK : TT_EDEVICE;
}
