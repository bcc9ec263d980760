// Wave-wide operations (64 lanes) of the token operators' kernels, and what those kernels share: reductions over a wave or a
// workgroup, 16-byte vectors at any element's alignment, bf16 values.  The host emulation build takes its stand-ins of the
// wave-wide operations from emu_wave.h.
#pragma once
#include <cstdint>
#include "tt_device.h"
#include "tt_bf16.h"
#ifdef TT_HOST_EMULATION
#include "emu_wave.h"
#define TT_GLOBAL
#define TT_CONSTANT
#else
// Memory that is not LDS, said so: for a pointer out of a table the compiler makes accesses that could be either, which count as
// both and are waited for as such.
#define TT_GLOBAL __attribute__((address_space(1)))
// Memory that nothing writes while the kernel runs: a value at an address that all lanes share comes as a scalar, and is waited
// for apart from the vectors on their way.
#define TT_CONSTANT __attribute__((address_space(4)))
namespace tt {
namespace wave {

__device__ __forceinline__ uint32_t shfl_xor(uint32_t v, int mask) { return (uint32_t)__shfl_xor((int)v, mask, 64); }
__device__ __forceinline__ double shfl_xor(double v, int mask) { return __shfl_xor(v, mask, 64); }
__device__ __forceinline__ uint32_t shfl_up(uint32_t v, int by) { return (uint32_t)__shfl_up((int)v, by, 64); }
__device__ __forceinline__ uint32_t read_lane(uint32_t v, int from) { return (uint32_t)__builtin_amdgcn_readlane((int)v, from); }
__device__ __forceinline__ uint64_t ballot(bool p) { return __ballot(p); }
// integer counter in LDS (the order of additions does not matter)
__device__ __forceinline__ void lds_add(uint32_t *p, uint32_t v) { atomicAdd(p, v); }
// LDS accesses of the wave's lanes before this are done, and those after it not begun
__device__ __forceinline__ void fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// The compiler takes v for a new value from here on: what it worked out from v before is worked out again instead of being kept
// (a row that waits in registers as 16 bits a value must not wait as 32).
template <typename V> __device__ __forceinline__ void forget(V &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void forget_uniform(uint32_t &v) { asm volatile("" : "+s"(v)); }
// 2^x (1 ulp; what lies below 2^-126 is 0)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// v of the lane that a data-parallel-primitive control names, `other` where it names none
template <int CTRL, int ROWS> __device__ __forceinline__ float moved(float v, float other)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(other), (int)__float_as_uint(v), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t v, uint32_t other)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)other, (int)v, CTRL, ROWS, 0xf, false);
}
// v combined over the wave, in every lane: up the rows of 16 lanes (shifts by 1, 2, 4, 8), then from row to row (the last lane of
// a row to the next one, of the lower half to the upper).  No trip through LDS; the order of additions is fixed.
template <typename V, class F> __device__ __forceinline__ V combined(V v, V none, F &&f)
{
    v = f(v, moved<0x111, 0xf>(v, none));
    v = f(v, moved<0x112, 0xf>(v, none));
    v = f(v, moved<0x114, 0xf>(v, none));
    v = f(v, moved<0x118, 0xf>(v, none));
    v = f(v, moved<0x142, 0xa>(v, none));
    v = f(v, moved<0x143, 0xc>(v, none));
    if constexpr (sizeof(V) == 4 && !__is_same(V, uint32_t)) return __uint_as_float(read_lane(__float_as_uint(v), 63));
    else return read_lane(v, 63);
}

// the low bytes of four words, a's first
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(d, c, 0x0c0c0400u) << 16 | __builtin_amdgcn_perm(b, a, 0x0c0c0400u);
}

} // namespace wave
} // namespace tt
#endif

namespace tt {

// a value that all lanes of a wave hold, in a scalar register
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

__device__ __forceinline__ uint64_t uniform(uint64_t v) { return (uint64_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v); }

__device__ __forceinline__ float wave_max(float v) { return wave::combined(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float v) { return wave::combined(v, 0.0f, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) { return wave::combined(v, 0u, [](uint32_t a, uint32_t b) { return a + b; }); }

// ---- 16-byte vectors that begin at any element: rows of odd length begin anywhere, and the memory system takes a 16-byte
// access at any address (the compiler splits it where a target does not)
template <int ALIGN> struct Vec16;
template <> struct Vec16<2> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Vec16<4> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T> __device__ __forceinline__ u32x4 load16(const T *p)
{
    typedef typename Vec16<sizeof(T)>::type V;
    const V v = *(const TT_GLOBAL V *)p;
    return u32x4{v.x, v.y, v.z, v.w};
}
template <typename T> __device__ __forceinline__ void store16(T *p, u32x4 v)
{
    typedef typename Vec16<sizeof(T)>::type V;
    *(TT_GLOBAL V *)p = v;
}

template <typename T> __device__ __forceinline__ void store16_once(T *p, u32x4 v) // (nobody reads it soon: no place in the caches)
{
    typedef typename Vec16<sizeof(T)>::type V;
    __builtin_nontemporal_store((V)v, (TT_GLOBAL V *)p);
}
template <typename T> __device__ __forceinline__ T load_scalar(const T *p) { return *(const TT_CONSTANT T *)p; }
template <typename T> __device__ __forceinline__ T load1(const T *p) { return *(const TT_GLOBAL T *)p; }
template <typename T> __device__ __forceinline__ void store1(T *p, T v) { *(TT_GLOBAL T *)p = v; }

// ---- element types: bf16 travels as its 16 bits
__device__ __forceinline__ float bf16_lo(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }
__device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float to_float(float v) { return v; }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t from_float<uint16_t>(float v) { return (uint16_t)f32_to_bf16_bits(v); }

// a 16-byte vector as 4 or 8 floats, and back (round to nearest even)
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);
__device__ __forceinline__ void unpack16(u32x4 v, float (&f)[8], uint16_t)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(v[i]); f[2 * i + 1] = bf16_hi(v[i]); }
}
__device__ __forceinline__ void unpack16(u32x4 v, float (&f)[4], float)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
}
__device__ __forceinline__ u32x4 pack16(const float (&f)[8], uint16_t)
{
    return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}
__device__ __forceinline__ u32x4 pack16(const float (&f)[4], float)
{
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
}

} // namespace tt
