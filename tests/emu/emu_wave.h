// Host stand-ins for the wave-wide operations of csrc/tt_wave.h, in lock step (emu_lockstep.h): every lane that has not ended
// takes part, as on the device where all 64 are active.
#pragma once
#ifndef TT_EMU_LOCKSTEP
#error "the token operators' kernels read what other lanes wrote: lock-step emulation only"
#endif

inline uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)(((uint64_t)a * b) >> 32); }

namespace tt {
namespace wave {

// each lane gives a word and gets the word of lane from(lane)
template <class F> inline uint32_t exchange(int kind, uint32_t v, F &&from)
{
    emu::WaveState &w = emu::my_wave();
    const int l = emu::lane();
    std::memcpy(&w.fa[l], &v, 4);
    emu::wave_collective(kind, [](emu::WaveState &s) { std::memcpy(s.fb, s.fa, sizeof(s.fa)); });
    uint32_t r;
    std::memcpy(&r, &w.fb[from(l)], 4);
    return r;
}
inline uint32_t shfl_xor(uint32_t v, int mask) { return exchange(10, v, [&](int l) { return l ^ mask; }); }
inline float shfl_xor(float v, int mask) { return __uint_as_float(shfl_xor(__float_as_uint(v), mask)); } // (combined)
inline double shfl_xor(double v, int mask)
{
    uint32_t h[2];
    std::memcpy(h, &v, 8);
    h[0] = shfl_xor(h[0], mask);
    h[1] = shfl_xor(h[1], mask);
    std::memcpy(&v, h, 8);
    return v;
}
inline uint32_t shfl_up(uint32_t v, int by) { return exchange(11, v, [&](int l) { return l >= by ? l - by : l; }); }
inline uint32_t read_lane(uint32_t v, int from) { return exchange(12, v, [&](int) { return from; }); }
inline uint64_t ballot(bool p)
{
    uint64_t m = 0;
    emu::WaveState &w = emu::my_wave();
    const int l = emu::lane();
    w.fa[l] = p ? 1.0f : 0.0f;
    emu::wave_collective(13, [](emu::WaveState &s) { std::memcpy(s.fb, s.fa, sizeof(s.fa)); });
    for (int i = 0; i < emu::kWave; ++i) m |= (uint64_t)(w.fb[i] != 0.0f) << i;
    return m;
}
template <typename V, class F> inline V combined(V v, V, F &&f)
{
    for (int m = 1; m < 64; m <<= 1) v = f(v, shfl_xor(v, m));
    return v;
}
inline uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return (a & 255u) | (b & 255u) << 8 | (c & 255u) << 16 | d << 24; }
inline void lds_add(uint32_t *p, uint32_t v) { *p += v; }
inline void fence() { emu::wave_sync(); }
template <typename V> inline void forget(V &) {}
inline void forget_uniform(uint32_t &) {}
inline float exp2_fast(float x) { return std::exp2(x); }

} // namespace wave
} // namespace tt
