// Host emulation of the matrix unit and of the transposing LDS read, as the gradient kernel uses them: the lanes of a
// wavefront lay their operands out, meet, and work on one another's.
#pragma once
#include <hip/hip_runtime.h>

namespace dgs {

static inline float emu_bf16(uint32_t word, int half)
{
    return __uint_as_float(half ? word & 0xFFFF0000u : word << 16);
}

static f32x16 matrix_unit(u32x4 a, u32x4 b, f32x16 c)
{
    static uint32_t A[1024][4], B[1024][4];
    const uint32_t t = threadIdx.x, first = t & ~63u, lane = t & 63u;
    for (int i = 0; i < 4; ++i) {
        A[t][i] = a[i];
        B[t][i] = b[i];
    }
    __builtin_amdgcn_wave_barrier();
    for (uint32_t j = 0; j < 16; ++j) {
        const uint32_t m = (j & 3u) + 8 * (j >> 2) + 4 * (lane >> 5), n = lane & 31u;
        for (uint32_t k = 0; k < 16; ++k) {
            const uint32_t half = first + 32 * (k >> 3), w = (k & 7u) >> 1;
            c[j] += emu_bf16(A[half + m][w], k & 1) * emu_bf16(B[half + n][w], k & 1);
        }
    }
    __builtin_amdgcn_wave_barrier();
    return c;
}

static u32x2 read_turned(const uint16_t *p)
{
    static const uint16_t *at[1024];
    const uint32_t t = threadIdx.x, first = t & ~15u, lane = t & 15u;
    at[t] = p;
    __builtin_amdgcn_wave_barrier();
    uint16_t v[4];
    for (uint32_t r = 0; r < 4; ++r) v[r] = at[first + 4 * r + (lane >> 2)][lane & 3u];
    __builtin_amdgcn_wave_barrier();
    u32x2 o;
    o[0] = v[0] | (uint32_t)v[1] << 16;
    o[1] = v[2] | (uint32_t)v[3] << 16;
    return o;
}

}  // namespace dgs
