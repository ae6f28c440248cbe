// Matrix products of 16-bit operands, a tile of the result to a workgroup: c[m][n] = sum_k a[m][k] b[n][k] on the matrix units,
// summed in fp32.
//
// An operand lies in memory with the summed index k inside (rows of k: "straight") or outside (rows of m or n: "turned").
// Either way 64 k of it are staged as they lie, by loads that go from memory to LDS without passing through registers, and a
// turned one is turned on its way out by the transposing LDS read.  What such a load writes is fixed -- lane l's 16 bytes
// behind lane l - 1's -- so the order that keeps LDS banks apart is made by what the lanes ask for: 16-byte pieces of a row
// are exchanged among one another.  A lane that asks for nothing there is (a row or a k beyond the matrix) asks beyond the
// buffer's end and gets zeros.
//
// An operand may be held in two parts, whose sum it is (22 bits of a value as two halves).  The product then goes over the
// same k once for every pair of parts that counts, as if the sum were so much longer.
#pragma once
#include "dgs_rows.h"

namespace dgs {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));      // eight 16-bit values of a lane
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t NOWHERE = 0x80000000u;      // an offset beyond every buffer

#ifdef DGS_HOST_EMULATION
}  // namespace dgs
#include "emu_product.h"
namespace dgs {
#else
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// c += a b: 32 x 32, 16 deep.  Lane l holds row (column) l % 32 of a (b), values 8 (l / 32) to 8 (l / 32) + 7 of the sum's
// index, and column l % 32 of c, rows (j % 4) + 8 (j / 4) + 4 (l / 32).
template <class E> __device__ __forceinline__ f32x16 matrix_unit_of(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (__is_same(E, f16))
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Sixteen lanes read 8 bytes each, four 16-bit values of row j / 4 from column 4 (j % 4) on; lane j gets column j of the four rows.
__device__ __forceinline__ u32x2 read_turned(const uint16_t *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

// Memory that a workgroup's loads start from.
typedef i32x4 Window;
__device__ __forceinline__ Window window_at(const void *p)
{
    const uint64_t a = (uint64_t)p;
    Window w;
    w.x = (int)uniform((uint32_t)a);
    w.y = (int)(uniform((uint32_t)(a >> 32)) & 0xFFFFu);
    w.z = (int)0x7FFFFFFF;
    w.w = 0x00020000;
    return w;
}
// 16 bytes from `offset` on into LDS: lane l's at `to` + 16 l.  Nothing waits; loads_done() does.
__device__ __forceinline__ void load_to_lds(Window w, uint32_t offset, uint16_t *to)
{
    const uint32_t at = uniform((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(offset), "s"(w) : "memory");
}
template <int LEFT> __device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory"); }
#endif

// One side of a product.
struct Side {
    const uint16_t *part[2];
    uint64_t stride;      // elements from row to row, a multiple of 8; rows start at multiples of 16 bytes
    uint32_t size;        // m or n
};

constexpr uint32_t PRODUCT_STEP = 64;

// Loads of one operand: WIDTH of its m (or n) and a step of k, by WAVES wavefronts.
template <uint32_t WIDTH, bool TURNED, uint32_t WAVES> struct Staged {
    static constexpr uint32_t LOADS = WIDTH * PRODUCT_STEP / 8 / 64 / WAVES;
    // turned: pieces of a row (its columns m), exchanged so that the four rows that 32 lanes read 64 bytes of lie in different
    // banks; straight: pieces of a row (its k), exchanged so that 16 rows' pieces of the same k do
    static constexpr uint32_t PIECES = TURNED ? WIDTH / 8 : PRODUCT_STEP / 8;
    static __device__ __forceinline__ uint32_t at(uint32_t row, uint32_t piece)
    {
        return row * PIECES * 8 + ((TURNED ? piece ^ ((row & 3u) << 2) : piece ^ ((row >> 1) & 7u)) << 3);
    }
    uint32_t offset[LOADS], k[LOADS];

    __device__ __forceinline__ void plan(const Side &s, uint32_t first)
    {
        const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6);
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t slot = (i * WAVES + wave) * 64 + lane, row = slot / PIECES;
            const uint32_t piece = ((at(row, slot % PIECES) >> 3) % PIECES);      // (an exchange undoes itself)
            const uint32_t outer = TURNED ? first + piece * 8 : first + row;
            offset[i] = outer < s.size ? (uint32_t)(row * s.stride + piece * 8) * 2u : NOWHERE;
            k[i] = TURNED ? row : piece * 8;
        }
    }
    __device__ __forceinline__ void load(const Side &s, uint32_t part, uint32_t first, uint32_t k0, uint32_t k_end, uint16_t *lds) const
    {
        const uint32_t wave = uniform(threadIdx.x >> 6);
        const Window w = window_at((part ? s.part[1] : s.part[0]) + (TURNED ? k0 * s.stride + first : first * s.stride + k0));
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) load_to_lds(w, k0 + k[i] < k_end ? offset[i] : NOWHERE, lds + (i * WAVES + wave) * 512);
    }
    // The operand of one matrix instruction: 32 of m from `m` on, k from 16 s to 16 s + 15.
    static __device__ __forceinline__ u32x4 fragment(const uint16_t *lds, uint32_t m, uint32_t s)
    {
        const uint32_t lane = lane_id();
        if constexpr (TURNED) {
            const uint32_t turn_k = ((lane >> 5) << 3) + ((lane & 15u) >> 2), turn_c = ((lane >> 4) & 1u) * 2u + ((lane & 3u) >> 1);
            u32x4 f;
#pragma unroll
            for (uint32_t r = 0; r < 2; ++r) {
                const u32x2 v = read_turned(lds + at(16 * s + turn_k + 4 * r, (m >> 3) + turn_c) + (lane & 1u) * 4);
                f[2 * r] = v.x;
                f[2 * r + 1] = v.y;
            }
            return f;
        } else {
            return *(const u32x4 *)(lds + at(m + (lane & 31u), 2 * s + (lane >> 5)));
        }
    }
};

// Row of sum r of a lane in a 32 x 32 square, its column being lane % 32: row_in_square(r), plus 4 in the upper 32 lanes.
__device__ __forceinline__ constexpr uint32_t row_in_square(uint32_t r) { return (r & 3u) + 8 * (r >> 2); }
__device__ __forceinline__ uint32_t square_row(uint32_t r) { return row_in_square(r) + 4 * (lane_id() >> 5); }

// The pairs of parts that a product goes over, two bits each: the first operand's part, and twice the second's.
constexpr uint32_t ONE_PAIR = 0x1, FIRST_IN_TWO = 0x2, BOTH_IN_TWO = 0x3;
__device__ __forceinline__ uint32_t pairs_of(uint32_t kind) { return kind == ONE_PAIR ? 1u : kind == FIRST_IN_TWO ? 2u : 3u; }

template <class E, uint32_t M, uint32_t N, uint32_t WAVES_M, uint32_t WAVES_N, bool TURN_A, bool TURN_B> struct Product {
    static constexpr uint32_t WAVES = WAVES_M * WAVES_N, THREADS = WAVES * 64, I = M / 32 / WAVES_M, J = N / 32 / WAVES_N;
    typedef Staged<M, TURN_A, WAVES> A;
    typedef Staged<N, TURN_B, WAVES> B;
    // Behind the sums, LDS takes a part of them from each wavefront (by_rows, by_columns).
    static constexpr uint32_t ABOVE = I < 2 ? 1 : 2, ROW_PITCH = 32 * J + 4, COLUMN_PITCH = 32 * ABOVE + 4;
    static constexpr uint32_t PART = 32 * ROW_PITCH > 32 * J * COLUMN_PITCH ? 32 * ROW_PITCH : 32 * J * COLUMN_PITCH;
    union Lds {
        struct {
            uint16_t a[2][M * PRODUCT_STEP], b[2][N * PRODUCT_STEP];
        };
        float part[WAVES][PART];
    };
    typedef f32x16 Sums[I][J];

    // This wavefront's first m and n in the tile.
    static __device__ __forceinline__ uint32_t wave_m() { return uniform(threadIdx.x >> 6) / WAVES_N * (32 * I); }
    static __device__ __forceinline__ uint32_t wave_n() { return uniform(threadIdx.x >> 6) % WAVES_N * (32 * J); }

    // Sums over k from k_first (a multiple of 8) to k_end, over the pairs of parts of `kind`.
    static __device__ __forceinline__ void run(Lds &lds, const Side &a, const Side &b, uint32_t m0, uint32_t n0, uint32_t k_first,
                                               uint32_t k_end, uint32_t kind, Sums &sums)
    {
        A la;
        B lb;
        la.plan(a, m0);
        lb.plan(b, n0);
#pragma unroll
        for (uint32_t i = 0; i < I; ++i)
#pragma unroll
            for (uint32_t j = 0; j < J; ++j)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) sums[i][j][r] = 0.0f;
        const uint32_t per_pair = k_end > k_first ? (k_end - k_first + PRODUCT_STEP - 1) / PRODUCT_STEP : 0u;
        const uint32_t steps = per_pair * pairs_of(kind);
        const uint32_t wm = wave_m(), wn = wave_n();
        uint32_t next = 0, next_k = k_first, pair = 0;      // what is loaded next
        auto load = [&](uint32_t buf) {
            // pairs: first with first, second with first, first with second
            la.load(a, pair == 1, m0, next_k, k_end, lds.a[buf]);
            lb.load(b, pair == 2, n0, next_k, k_end, lds.b[buf]);
            next_k += PRODUCT_STEP;
            if (++next == per_pair) {
                next = 0;
                next_k = k_first;
                ++pair;
            }
        };
        if (steps) load(0);
        for (uint32_t step = 0; step < steps; ++step) {
            const uint32_t buf = step & 1u;
            loads_done<0>();
            __syncthreads();      // this step has arrived, and nobody reads the one before any more
            if (step + 1 < steps) load(buf ^ 1u);
#pragma unroll
            for (uint32_t s = 0; s < PRODUCT_STEP / 16; ++s) {
                u32x4 fa[I], fb[J];
#pragma unroll
                for (uint32_t j = 0; j < J; ++j) fb[j] = B::fragment(lds.b[buf], wn + 32 * j, s);
#pragma unroll
                for (uint32_t i = 0; i < I; ++i) fa[i] = A::fragment(lds.a[buf], wm + 32 * i, s);
#pragma unroll
                for (uint32_t i = 0; i < I; ++i)
#pragma unroll
                    for (uint32_t j = 0; j < J; ++j) sums[i][j] = matrix_unit_of<E>(fa[i], fb[j], sums[i][j]);
            }
        }
    }

    // The lanes hold a column of a square each, four rows together.  Memory wants rows: the sums go through LDS, a wavefront's own
    // part of it, and come back as eight values of a row.  look(p, m, n) for every p first (what has to be loaded, so that the loads are
    // in flight together), then take(p, m, n, v), m and n in the tile.
    static constexpr uint32_t PASSES = 2 * J;      // of by_rows, 32 rows
    template <class Look, class Take> static __device__ __forceinline__ void by_rows(Lds &lds, const Sums &sums, Look look, Take take)
    {
        const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6), wm = wave_m(), wn = wave_n();
        float *const mine = lds.part[wave];
        __syncthreads();      // nobody reads operands any more
#pragma unroll
        for (uint32_t i = 0; i < I; ++i) {
#pragma unroll
            for (uint32_t p = 0; p < PASSES; ++p) {
                const uint32_t at = p * 64 + lane;
                look(p, wm + 32 * i + at / (4 * J), wn + at % (4 * J) * 8);
            }
#pragma unroll
            for (uint32_t j = 0; j < J; ++j)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) mine[square_row(r) * ROW_PITCH + 32 * j + (lane & 31u)] = sums[i][j][r];
            meet();
#pragma unroll
            for (uint32_t p = 0; p < PASSES; ++p) {
                const uint32_t at = p * 64 + lane, row = at / (4 * J), c = at % (4 * J) * 8;
                float v[8];
#pragma unroll
                for (uint32_t k = 0; k < 2; ++k) {
                    const f32x4 w = *(const f32x4 *)(mine + row * ROW_PITCH + c + 4 * k);
                    v[4 * k] = w.x; v[4 * k + 1] = w.y; v[4 * k + 2] = w.z; v[4 * k + 3] = w.w;
                }
                take(p, wm + 32 * i + row, wn + c, v);
            }
            meet();
        }
    }
    // The same where the values are wanted by columns too: take(p, m, n, v, back) leaves at `back` what turn(m, n, v) gets as eight values
    // of a column, m to m + 7.
    template <class Look, class Take, class Turn> static __device__ __forceinline__ void by_rows(Lds &lds, const Sums &sums, Look look, Take take, Turn turn)
    {
        const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6), wm = wave_m(), wn = wave_n();
        float *const mine = lds.part[wave];
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < I; ++i) {
#pragma unroll
            for (uint32_t p = 0; p < PASSES; ++p) {
                const uint32_t at = p * 64 + lane;
                look(p, wm + 32 * i + at / (4 * J), wn + at % (4 * J) * 8);
            }
#pragma unroll
            for (uint32_t j = 0; j < J; ++j)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) mine[square_row(r) * ROW_PITCH + 32 * j + (lane & 31u)] = sums[i][j][r];
            meet();
#pragma unroll
            for (uint32_t p = 0; p < PASSES; ++p) {
                const uint32_t at = p * 64 + lane, row = at / (4 * J), c = at % (4 * J) * 8;
                float v[8], back[8];
                float *const here = mine + row * ROW_PITCH + c;
#pragma unroll
                for (uint32_t k = 0; k < 2; ++k) {
                    const f32x4 w = *(const f32x4 *)(here + 4 * k);
                    v[4 * k] = w.x; v[4 * k + 1] = w.y; v[4 * k + 2] = w.z; v[4 * k + 3] = w.w;
                }
                take(p, wm + 32 * i + row, wn + c, v, back);
#pragma unroll
                for (uint32_t k = 0; k < 2; ++k) {
                    f32x4 w;
                    w.x = back[4 * k]; w.y = back[4 * k + 1]; w.z = back[4 * k + 2]; w.w = back[4 * k + 3];
                    *(f32x4 *)(here + 4 * k) = w;
                }
            }
            meet();
#pragma unroll
            for (uint32_t p = 0; p < PASSES; ++p) {
                // four lanes a column, so that memory gets 32 values of it together
                const uint32_t at = p * 64 + lane, col = at >> 2, row = (at & 3u) * 8;
                float v[8];
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) v[k] = mine[(row + k) * ROW_PITCH + col];
                turn(wm + 32 * i + row, wn + col, v);
            }
            meet();
        }
    }
    // Eight values of a column, m to m + 7, in the same way: take(m, n, v).
    template <class Take> static __device__ __forceinline__ void by_columns(Lds &lds, const Sums &sums, Take take)
    {
        const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6), wm = wave_m(), wn = wave_n();
        float *const mine = lds.part[wave];
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < I; i += ABOVE) {
#pragma unroll
            for (uint32_t above = 0; above < ABOVE; ++above)
#pragma unroll
                for (uint32_t j = 0; j < J; ++j)
#pragma unroll
                    for (uint32_t g = 0; g < 4; ++g) {
                        f32x4 w;
                        w.x = sums[i + above][j][4 * g]; w.y = sums[i + above][j][4 * g + 1];
                        w.z = sums[i + above][j][4 * g + 2]; w.w = sums[i + above][j][4 * g + 3];
                        *(f32x4 *)(mine + (32 * j + (lane & 31u)) * COLUMN_PITCH + 32 * above + square_row(4 * g)) = w;
                    }
            meet();
#pragma unroll
            for (uint32_t p = 0; p < 2 * J * ABOVE; ++p) {
                const uint32_t at = p * 64 + lane, n = at / (4 * ABOVE), m = at % (4 * ABOVE) * 8;
                float v[8];
#pragma unroll
                for (uint32_t k = 0; k < 2; ++k) {
                    const f32x4 w = *(const f32x4 *)(mine + n * COLUMN_PITCH + m + 4 * k);
                    v[4 * k] = w.x; v[4 * k + 1] = w.y; v[4 * k + 2] = w.z; v[4 * k + 3] = w.w;
                }
                take(wm + 32 * i + m, wn + n, v);
            }
            meet();
        }
    }
    // What lanes of a wavefront have written to LDS is there for the others.
    static __device__ __forceinline__ void meet()
    {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
};

// Workgroup `block` of `total`, of which neighbours go to different dies: every die gets a run of the tiles.
__device__ __forceinline__ uint32_t tile_of_block(uint32_t block, uint32_t total)
{
    const uint32_t die = block & 7u;
    return die * (total >> 3) + min(die, total & 7u) + (block >> 3);
}

// A value in two halves (22 bits).
__device__ __forceinline__ void halves_of(float v, f16 &hi, f16 &lo)
{
    hi = (f16)v;
    lo = (f16)(v - (float)hi);
}
__device__ __forceinline__ uint32_t bits_of(f16 a, f16 b)
{
    uint16_t x, y;
    __builtin_memcpy(&x, &a, 2);
    __builtin_memcpy(&y, &b, 2);
    return x | (uint32_t)y << 16;
}

// Eight values as halves, in one part or two.
__device__ __forceinline__ void halves8(const float (&v)[8], u32x4 &hi, u32x4 &lo)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f16 a, b, c, d;
        halves_of(v[2 * i], a, b);
        halves_of(v[2 * i + 1], c, d);
        hi[i] = bits_of(a, c);
        lo[i] = bits_of(b, d);
    }
}

// Sections of a workspace, one after another, each from a multiple of 256 bytes behind its start on.  (Nothing is reached through
// what a null workspace gives: its sizes count.)
struct Sections {
    uintptr_t base;
    uint64_t used;
    void *take(uint64_t bytes)
    {
        void *const p = (void *)(base + used);
        used += (bytes + 255) & ~255ull;
        return p;
    }
};

}  // namespace dgs
