// Host build of the library (lock-step emulation): csrc/fc8.hip.
#define TT_HOST_EMULATION 1
#include <cstdint>
#include "tt_device.h"

// v_mfma_i32_16x16x64_i8: A: row lane % 16, k = 16 (lane / 16) + 0..15; B: column lane % 16, the same k; C, D: column lane % 16, row
// 4 (lane / 16) + r for register r; sums modulo 2^32
namespace emu {
template <class V> inline V mfma_16x16x64_i8(V a, V b, V c)
{
    static_assert(sizeof(V) == 16, "operand registers of v_mfma_i32_16x16x64_i8");
    WaveState &w = my_wave();
    const int l = lane();
    std::memcpy(w.a[l], &a, 16);
    std::memcpy(w.b[l], &b, 16);
    std::memcpy(w.c[l], &c, 16);
    wave_collective(20, [](WaveState &v) {
        if (v.live != kWave) die("MFMA in a wave with ended lanes");
        for (int ln = 0; ln < kWave; ++ln)
            for (int r = 0; r < 4; ++r) {
                const int i = 4 * (ln / 16) + r, j = ln % 16;
                uint32_t s;
                std::memcpy(&s, &v.c[ln][r], 4);
                for (int k = 0; k < 64; ++k) {
                    const int8_t x = reinterpret_cast<const int8_t *>(v.a[i + 16 * (k / 16)])[k % 16], y = reinterpret_cast<const int8_t *>(v.b[j + 16 * (k / 16)])[k % 16];
                    s += (uint32_t)((int32_t)x * (int32_t)y);
                }
                std::memcpy(&v.c[ln][r], &s, 4);
            }
    });
    std::memcpy(&c, w.c[l], 16);
    return c;
}
} // namespace emu
#define __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, x, y, z) emu::mfma_16x16x64_i8(a, b, c)

namespace tt {
namespace {
alignas(16) thread_local char smem8[160 * 1024]; // what the kernels' `extern __shared__` array refers to here
}
} // namespace tt
#include "fc8.hip"
static const int g_registered = emu_register_lds(tt::smem8, sizeof(tt::smem8));
