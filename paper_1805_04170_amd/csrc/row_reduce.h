// Sums and maxima over the lanes that hold a row between them: a group of 2^n lanes of a wave (WAVE), or a workgroup.
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

// LDS of a row's reductions.  Two sets in turn, so that one barrier a reduction is enough: a set is written again only after the
// barrier of the reduction between, which all threads pass after they have read it.
template <int N> struct RowScratch { double v[2][N][kMostWaves]; };

// N values at a time combined over the row, value i by F[i]; `turn` alternates from call to call.
template <bool WAVE, typename V, class... F> struct RowReduce {
    static constexpr int N = sizeof...(F);
    template <class S> static __device__ __forceinline__ void run(V (&v)[N], uint32_t lanes, S &scratch, uint32_t turn)
    {
        int i = 0;
        ((v[i] = over_lanes<F>(v[i], WAVE ? lanes : 64u), ++i), ...);
        if constexpr (!WAVE) {
            const uint32_t waves = lanes >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
            if (waves == 1) return;
            for (i = 0; i < N; ++i) // (all lanes of a wave have the same)
                if (lane == 0) reinterpret_cast<V *>(scratch.v[turn & 1][i])[wave] = v[i];
            __syncthreads();
            i = 0;
            ((v[i] = joined<F>(reinterpret_cast<const V *>(scratch.v[turn & 1][i]), waves), ++i), ...);
        }
    }
    template <class G> static __device__ __forceinline__ V joined(const V *of_wave, uint32_t waves)
    {
        // lane l takes wave l % 16's (0 where there is none), sixteen lanes together all
        const uint32_t l = threadIdx.x & (kMostWaves - 1);
        return over_lanes<G>(l < waves ? of_wave[l] : V(0), (uint32_t)kMostWaves);
    }
};

// How a launch lays its rows out: `lanes` threads a row.
struct RowLaunch {
    bool wave;
    int vectors;          // of a thread: 1, 2, 4;  0: rows too long for registers
    uint32_t lanes, block;
    uint32_t at_once;     // rows of a workgroup at a time
};
inline RowLaunch row_launch(const RowShape &r)
{
    if (r.units <= 64) {
        uint32_t lanes = 1;
        while (lanes < r.units) lanes <<= 1;
        return {true, 1, lanes, kWaveBlock, kWaveBlock / lanes};
    }
    for (int v = 1; v <= 4; v *= 2) {
        const uint32_t lanes = ((r.units + v - 1) / v + 63) / 64 * 64;
        if (lanes <= kMostThreads) return {false, v, lanes, lanes, 1};
    }
    return {false, 0, kMostThreads, kMostThreads, 1};
}

// kinds of memory access
enum { kPlain = 0, kCut = 1, kNarrow = 2 };

} // namespace tt
