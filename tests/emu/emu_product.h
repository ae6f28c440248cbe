// Host emulation of the product kernels' builtins: matrix units of both 16-bit types, the transposing LDS read, and the load
// from memory to LDS, whose lanes' 16 bytes lie one behind the other and which is zeros beyond the buffer's end.
#pragma once
#include "emu_matrix.h"

namespace dgs {

struct float2 { float x, y; };
static inline float2 make_float2(float x, float y) { return float2{x, y}; }

static inline float emu_f16(uint32_t word, int half)
{
    const uint16_t h = (uint16_t)(half ? word >> 16 : word);
    _Float16 f;
    memcpy(&f, &h, 2);
    return (float)f;
}

template <class E> static f32x16 matrix_unit_of(u32x4 a, u32x4 b, f32x16 c)
{
    if (__is_same(E, bf16)) return matrix_unit(a, b, c);
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
            c[j] += emu_f16(A[half + m][w], k & 1) * emu_f16(B[half + n][w], k & 1);
        }
    }
    __builtin_amdgcn_wave_barrier();
    return c;
}

struct Window { const char *p; uint32_t bytes; };
static inline Window window_at(const void *p, uint32_t bytes) { return Window{(const char *)p, bytes}; }
typedef uint16_t *LdsPlace;
static inline LdsPlace lds_place(uint16_t *p) { return p; }
static inline void load_to_lds(Window w, uint32_t offset, LdsPlace to, uint32_t behind)
{
    char *const p = (char *)to + behind + 16 * (threadIdx.x & 63u);
    if (offset >= w.bytes) memset(p, 0, 16);
    else memcpy(p, w.p + offset, 16);
}
template <int LEFT> static inline void loads_meet() { __syncthreads(); }

}  // namespace dgs
