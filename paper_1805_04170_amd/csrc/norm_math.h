// What the kernels that take a row's root mean square share.
#pragma once
#include <cmath>
#include "row_reduce.h"

namespace tt {

// Squares of fp32 values may leave fp32.  Rows whose mean of squares does not lie well inside it (squares below 2^-126 lose bits, which
// a mean of 2^-80 does not notice) are summed again as values times a power of two, which rounds nothing.
__device__ __forceinline__ bool fits_fp32(float mean) { return mean >= 0x1p-80f && mean < 0x1p90f; }
__device__ __forceinline__ float factor_for(float mean) { return mean < 1.0f ? 0x1p80f : 0x1p-80f; }
__device__ __forceinline__ float scaled_mean(float sum, float per_col, float eps, float factor) { return sum * per_col + eps * factor * factor; }
// 1 / sqrt(mean) (1 ulp); NaN where the row held an infinity
__device__ __forceinline__ float inverse_root(float mean)
{
#ifdef TT_HOST_EMULATION
    const float r = 1.0f / sqrtf(mean);
#else
    const float r = __builtin_amdgcn_rsqf(mean);
#endif
    return mean < __builtin_inff() ? r : __builtin_nanf("");
}
__device__ __forceinline__ double inverse_root_wide(double mean) // (finite values of fp32 have a finite sum in 64 bits)
{
    return mean <= 0x1p300 ? 1.0 / sqrt(mean) : (double)__builtin_nanf("");
}

// R + X in the tensors' type
template <typename T> __device__ __forceinline__ u32x4 added(u32x4 x, u32x4 r)
{
    constexpr uint32_t EV = kVec<T>;
    float f[EV], g[EV];
    unpack16(x, f, T());
    unpack16(r, g, T());
#pragma unroll
    for (uint32_t e = 0; e < EV; ++e) f[e] += g[e];
    return pack16(f, T());
}

} // namespace tt
