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
// same k once for every pair of parts that counts, as if the sum were so much longer.  Second parts may be held times 2^LOW: the
// smallest of a half's numbers then cuts off 2^LOW times less.  Pairs with a second part go first, and what they sum to is divided once.
#pragma once
#include "dgs_rows.h"

namespace dgs {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));      // eight 16-bit values of a lane
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t NOWHERE = 0x80000000u, ANYWHERE = 0x7FFFFFFFu;      // an offset beyond every buffer, and the largest buffer

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

// Memory that a workgroup's loads start from, and how much of it there is: beyond it they get zeros.
typedef i32x4 Window;
__device__ __forceinline__ Window window_at(const void *p, uint32_t bytes)
{
    const uint64_t a = (uint64_t)p;
    Window w;
    w.x = (int)uniform((uint32_t)a);
    w.y = (int)(uniform((uint32_t)(a >> 32)) & 0xFFFFu);
    w.z = (int)uniform(bytes);
    w.w = 0x00020000;
    return w;
}
// Where in LDS a wavefront's loads go.
typedef uint32_t LdsPlace;
__device__ __forceinline__ LdsPlace lds_place(uint16_t *p) { return uniform((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)p); }
// 16 bytes from `offset` on into LDS: lane l's `behind` + 16 l bytes behind `to`.  Nothing waits; loads_meet() does.  (The compiler keeps
// nothing in m0, and warns that it would not save it; named, nothing of its own that sets and uses m0 is moved across.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(Window w, uint32_t offset, LdsPlace to, uint32_t behind)
{
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(w), "s"(behind) : "memory", "scc", "m0");
}
#pragma clang diagnostic pop
// Every wavefront's loads but its last LEFT have arrived, and what was read before has been.
template <int LEFT> __device__ __forceinline__ void loads_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory"); }
#endif

// One side of a product.
struct Side {
    const uint16_t *part[2];
    uint64_t stride;      // elements from row to row, a multiple of 8; rows start at multiples of 16 bytes
    uint32_t size;        // m or n
};

constexpr uint32_t PRODUCT_STEP = 64;      // of k, staged at a time

// Loads of one operand: WIDTH of its m (or n) and a step of k, by WAVES wavefronts.
template <uint32_t WIDTH, bool TURNED, uint32_t WAVES, uint32_t STEP> struct Staged {
    static constexpr uint32_t LOADS = WIDTH * STEP / 8 / 64 / WAVES;
    // turned: pieces of a row (its columns m), exchanged so that the four rows that 32 lanes read 64 bytes of lie in different
    // banks; straight: pieces of a row (its k), exchanged so that 16 rows' pieces of the same k do
    static constexpr uint32_t PIECES = TURNED ? WIDTH / 8 : STEP / 8;
    static __device__ __forceinline__ uint32_t at(uint32_t row, uint32_t piece)
    {
        return row * PIECES * 8 + ((!TURNED ? piece ^ ((row >> 1) & 7u) : PIECES == 8 ? piece ^ ((row & 2u) << 1) : piece ^ ((row & 3u) << 2)) << 3);
    }
    uint32_t offset[LOADS], k;      // (straight: the k that a lane loads is the same in all its loads)
    Window from;

    __device__ __forceinline__ void plan(const Side &s, uint32_t first)
    {
        const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6);
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t slot = (i * WAVES + wave) * 64 + lane, row = slot / PIECES;
            const uint32_t piece = ((at(row, slot % PIECES) >> 3) % PIECES);      // (an exchange undoes itself)
            const uint32_t outer = TURNED ? first + piece * 8 : first + row;
            offset[i] = outer < s.size ? (uint32_t)(row * s.stride + piece * 8) * 2u : NOWHERE;
            if (i == 0) k = piece * 8;
        }
    }
    // Where a step's loads are from; `left` of k are there.  (Turned: a row of k that is not there lies beyond the window.)
    __device__ __forceinline__ void step(const Side &s, uint32_t part, uint32_t first, uint32_t k0, uint32_t left)
    {
        const uint64_t bytes = TURNED ? left * s.stride * 2u : (uint64_t)ANYWHERE;
        from = window_at((part ? s.part[1] : s.part[0]) + (TURNED ? k0 * s.stride + first : first * s.stride + k0),
                         bytes < ANYWHERE ? (uint32_t)bytes : ANYWHERE);
        inside = k < left;
    }
    bool inside;
    // (`lds`: this wavefront's place in the first stage)
    __device__ __forceinline__ void load(uint32_t i, LdsPlace lds, uint32_t stage) const
    {
        load_to_lds(from, TURNED || inside ? offset[i] : NOWHERE, lds, stage * (WIDTH * STEP * 2) + i * WAVES * 1024);
    }
    static_assert(TURNED || PIECES == 8, "the exchange is of eight pieces");
    static_assert(LOADS > 0 && (TURNED || WAVES * 64 / PIECES % 16 == 0), "whole loads, of one k");
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

// Nothing is moved across this by the compiler, which would put LDS reads right before what waits for them.
__device__ __forceinline__ void in_order()
{
#ifndef DGS_HOST_EMULATION
    __builtin_amdgcn_sched_barrier(0);
#endif
}

template <class E, uint32_t M, uint32_t N, uint32_t WAVES_M, uint32_t WAVES_N, bool TURN_A, bool TURN_B, uint32_t STAGES, uint32_t STEP = PRODUCT_STEP, uint32_t LOW = 0> struct Product {
    static constexpr uint32_t WAVES = WAVES_M * WAVES_N, THREADS = WAVES * 64, I = M / 32 / WAVES_M, J = N / 32 / WAVES_N;
    typedef Staged<M, TURN_A, WAVES, STEP> A;
    typedef Staged<N, TURN_B, WAVES, STEP> B;
    // Behind the sums, LDS takes a part of them from each wavefront (by_rows, by_columns).
    static constexpr uint32_t ABOVE = I < 2 ? 1 : 2, ROW_PITCH = 32 * J + 4, COLUMN_PITCH = 32 * ABOVE + 4;
    static constexpr uint32_t PART = 32 * ROW_PITCH > 32 * J * COLUMN_PITCH ? 32 * ROW_PITCH : 32 * J * COLUMN_PITCH;
    union Lds {
        struct {
            uint16_t a[STAGES][M * STEP], b[STAGES][N * STEP];
        };
        __attribute__((aligned(16))) float part[WAVES][PART];
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
        const uint32_t per_pair = k_end > k_first ? (k_end - k_first + STEP - 1) / STEP : 0u;
        const uint32_t pairs = pairs_of(kind), steps = per_pair * pairs;
        if (steps == 0) return;
        const uint32_t wm = wave_m(), wn = wave_n();
        // what is loaded next; behind the last step nothing, in as many loads
        uint32_t next = 0, next_k = k_first, pair = 0, to = 0;
        auto next_step = [&]() {
            // pairs: first with first, second with first, first with second (LOW: first with first is the last)
            const uint32_t left = pair < pairs ? k_end - next_k : 0u;
            la.step(a, pair == (LOW ? 0 : 1) && pairs > 1, m0, next_k, left);
            lb.step(b, pair == (LOW ? 1 : 2) && pairs > 2, n0, next_k, left);
            next_k += STEP;
            if (++next == per_pair) {
                next = 0;
                next_k = k_first;
                ++pair;
            }
        };
        constexpr uint32_t EACH = A::LOADS + B::LOADS, SLICES = STEP / 16, READS = I + J, SQUARES = I * J;
        const uint32_t wave = uniform(threadIdx.x >> 6);
        const LdsPlace place_a = lds_place(lds.a[0] + wave * 512), place_b = lds_place(lds.b[0] + wave * 512);
        auto load = [&](uint32_t l) {
            if (l < A::LOADS) la.load(l, place_a, to);
            else lb.load(l - A::LOADS, place_b, to);
        };
        u32x4 fa[2][I], fb[2][J];
        auto read = [&](uint32_t stage, uint32_t s, uint32_t r) {
            if (r < J) fb[s & 1][r] = B::fragment(lds.b[stage], wn + 32 * r, s);
            else fa[s & 1][r - J] = A::fragment(lds.a[stage], wm + 32 * (r - J), s);
        };
        // A slice of 16 k: its matrix instructions, and between them the reads of the next slice's operands (early: they have to be there when
        // this one ends) and, in a step's last slice, the loads of the step after next.  The order is as written.
        auto slice = [&](uint32_t s, uint32_t read_stage, bool loads) {
#pragma unroll
            for (uint32_t q = 0; q < SQUARES; ++q) {
                sums[q / J][q % J] = matrix_unit_of<E>(fa[s & 1][q / J], fb[s & 1][q % J], sums[q / J][q % J]);
                in_order();
                constexpr uint32_t FEW = SQUARES >= 2 * READS ? 1 : SQUARES >= READS ? 1 : (READS + SQUARES - 1) / SQUARES;
#pragma unroll
                for (uint32_t r = q * FEW; r < (q + 1) * FEW; ++r)
                    if (r < READS) read(read_stage, (s + 1) % SLICES, r);
                if (loads) {
#pragma unroll
                    for (uint32_t l = q * EACH / SQUARES; l < (q + 1) * EACH / SQUARES; ++l) load(l);
                }
                in_order();
            }
        };
#pragma unroll
        for (uint32_t s = 0; s < STAGES; ++s) {
            next_step();
#pragma unroll
            for (uint32_t l = 0; l < EACH; ++l) load(l);
            to = (to + 1) % STAGES;
        }
        loads_meet<(STAGES - 1) * EACH>();
#pragma unroll
        for (uint32_t r = 0; r < READS; ++r) read(0, 0, r);
        // (sums of second parts are divided behind them)
        const uint32_t second = LOW && pairs > 1 ? steps - per_pair : 0u;
        for (uint32_t step = 0, stage = 0; step < steps; ++step) {
            if constexpr (LOW > 0) {
                if (second && step == second) {
                    in_order();      // (so that this stays a branch: a choice between both for every sum of every step costs small tiles a tenth)
#pragma unroll
                    for (uint32_t i = 0; i < I; ++i)
#pragma unroll
                        for (uint32_t j = 0; j < J; ++j) sums[i][j] *= 1.0f / (1u << LOW);
                }
            }
#pragma unroll
            for (uint32_t s = 0; s + 1 < SLICES; ++s) slice(s, stage, false);
            next_step();
            // this wavefront has read all of the step, and the next one has arrived: everybody's part of it
            loads_meet<(STAGES - 2) * EACH>();
            const uint32_t following = (stage + 1) % STAGES;
            slice(SLICES - 1, following, true);
            to = stage = following;
        }
        loads_meet<0>();      // (the loads of nothing)
    }

    // The lanes hold a column of a square each, four rows together.  Memory wants rows: the sums go through LDS, a wavefront's own
    // part of it, and come back as eight values of a row.  look(p, m, n) for every p first (what has to be loaded, so that the loads are
    // in flight together), then take(p, m, n, v), m and n in the tile.
    // (Where a wavefront has 32 rows alone, look_early() is called before the sums are taken, and by_rows looks no more.)
    static constexpr uint32_t PASSES = 2 * J;      // of by_rows, 32 rows
    template <class Look> static __device__ __forceinline__ void look_early(Look look)
    {
        if constexpr (I == 1) {
#pragma unroll
            for (uint32_t p = 0; p < PASSES; ++p) {
                const uint32_t at = p * 64 + lane_id();
                look(p, wave_m() + at / (4 * J), wave_n() + at % (4 * J) * 8);
            }
        }
    }
    template <class Look, class Take> static __device__ __forceinline__ void by_rows(Lds &lds, const Sums &sums, Look look, Take take)
    {
        const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6), wm = wave_m(), wn = wave_n();
        float *const mine = lds.part[wave];
        sync();      // nobody reads operands any more
#pragma unroll
        for (uint32_t i = 0; i < I; ++i) {
            if constexpr (I > 1) {
#pragma unroll
                for (uint32_t p = 0; p < PASSES; ++p) {
                    const uint32_t at = p * 64 + lane;
                    look(p, wm + 32 * i + at / (4 * J), wn + at % (4 * J) * 8);
                }
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
    // The same, four values at a time, for results of four bytes: a load or store of the wavefront is whole rows of 32 J values.
    template <class Look, class Take> static __device__ __forceinline__ void by_fours(Lds &lds, const Sums &sums, Look look, Take take)
    {
        const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6), wm = wave_m(), wn = wave_n();
        float *const mine = lds.part[wave];
        sync();
#pragma unroll
        for (uint32_t i = 0; i < I; ++i) {
#pragma unroll
            for (uint32_t p = 0; p < 2 * PASSES; ++p) {
                const uint32_t at = p * 64 + lane;
                look(p, wm + 32 * i + at / (8 * J), wn + at % (8 * J) * 4);
            }
#pragma unroll
            for (uint32_t j = 0; j < J; ++j)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) mine[square_row(r) * ROW_PITCH + 32 * j + (lane & 31u)] = sums[i][j][r];
            meet();
#pragma unroll
            for (uint32_t p = 0; p < 2 * PASSES; ++p) {
                const uint32_t at = p * 64 + lane, row = at / (8 * J), c = at % (8 * J) * 4;
                f32x4 v = *(const f32x4 *)(mine + row * ROW_PITCH + c);
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
        sync();
#pragma unroll
        for (uint32_t i = 0; i < I; ++i) {
            if constexpr (I > 1) {
#pragma unroll
                for (uint32_t p = 0; p < PASSES; ++p) {
                    const uint32_t at = p * 64 + lane;
                    look(p, wm + 32 * i + at / (4 * J), wn + at % (4 * J) * 8);
                }
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
        sync();
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
    // The tile's wavefronts meet (one alone needs no barrier, which others of its workgroup that have ended would not reach).
    static __device__ __forceinline__ void sync()
    {
        if constexpr (WAVES == 1) meet();
        else __syncthreads();
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
constexpr uint32_t TILE_BAND = 4;
// Tile `at` of m_tiles x n_tiles: bands of TILE_BAND rows of tiles, column by column, so that the 32 tiles that a die works on at a time
// are about as many high as wide and share what they load in its L2.
struct TilePlace { uint32_t m, n; };
__device__ __forceinline__ TilePlace place_of_tile(uint32_t at, uint32_t m_tiles, uint32_t n_tiles)
{
    const uint32_t band = at / (TILE_BAND * n_tiles), first = band * TILE_BAND, high = min(m_tiles - first, TILE_BAND), in = at - first * n_tiles;
    return TilePlace{first + in % high, in / high};
}

__device__ __forceinline__ float half_value(uint16_t bits)
{
    f16 h;
    __builtin_memcpy(&h, &bits, 2);
    return (float)h;
}

// Eight values as halves, in two parts (22 bits of each), the second times 2^LOW.  (Values below 2^16 leave less than 2^5 to it.)
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
template <uint32_t LOW = 0> __device__ __forceinline__ void halves8(const float (&v)[8], u32x4 &hi, u32x4 &lo)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 w = {v[2 * i], v[2 * i + 1]};
        const f16x2 h = __builtin_convertvector(w, f16x2);
        f32x2 left = {w.x - (float)h.x, w.y - (float)h.y};
        if constexpr (LOW > 0) left = f32x2{left.x * (1u << LOW), left.y * (1u << LOW)};
        const f16x2 l = __builtin_convertvector(left, f16x2);
        hi[i] = __builtin_bit_cast(uint32_t, h);
        lo[i] = __builtin_bit_cast(uint32_t, l);
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

// ---------------------------------------------------------------------------
// host side: which tile
// ---------------------------------------------------------------------------

// 256 x 256 to eight wavefronts and 192 x 192 to four, one workgroup to a compute unit; 256 x 128 (steps of 32), 128 x 128 and
// 64 x 64 to four, two workgroups to a compute unit.
enum ProductTile { TILE_256, TILE_TALL, TILE_192, TILE_128, TILE_64, PRODUCT_TILES };
static inline uint32_t tile_high(int tile) { return tile <= TILE_TALL ? 256 : tile == TILE_192 ? 192 : tile == TILE_128 ? 128 : 64; }
static inline uint32_t tile_wide(int tile) { return tile == TILE_TALL ? 128 : tile_high(tile); }
static inline uint32_t tiles_of(uint32_t n, uint32_t size) { return n ? (n - 1) / size + 1 : 0; }

// Microseconds that `tiles` tiles of `steps` steps of 64 k take: what a tile takes besides its steps, and for a step with every
// compute unit's places taken and with one workgroup to a compute unit at most, as timed.  (4096 x 4096 squares on and below the
// diagonal, 64 steps, by card: 256 x 256 93 to 110 us, 192 x 192 79 to 91, 128 x 128 107 to 114, 64 x 64 163 to 170; four of 1024 x 1024, 192 steps: 230, 128, 141; five of 333 x 333, 48
// steps: 66, 33, 17; 30522 x 768 turned, 256 steps: 256 x 256 882, 256 x 128 775, 128 x 128 845.)
static inline float tile_time(int tile, uint64_t tiles, uint32_t steps)
{
    static constexpr struct { float besides, full, one; uint32_t places; } cost[PRODUCT_TILES] = {
        {10.0f, 1.9f, 1.2f, 256}, {6.0f, 2.0f, 1.0f, 512}, {8.0f, 1.2f, 0.85f, 256}, {5.0f, 1.12f, 0.66f, 512}, {3.5f, 0.5f, 0.3f, 512}};
    const auto &c = cost[tile];
    const uint64_t rounds = tiles / c.places, rest = tiles % c.places;
    float us = (float)rounds * (c.besides + c.full * (float)steps);
    if (rest) {
        // (one to a compute unit: the clock falls as more of the chip multiplies)
        const float step = rest > 256 ? c.full : c.places > 256 ? c.one : c.one + (c.full - c.one) * (float)rest / 256.0f;
        us += c.besides + step * (float)steps;
    }
    return us;
}
// The tile that should take the least time; tiles(high, wide): how many of them there are.  `more`: TILE_TALL or TILE_192 where that
// is there too.
template <class Tiles> static int product_tile(Tiles tiles, uint32_t steps, int more, float &least)
{
    int best = TILE_256;
    for (int t = 0; t < PRODUCT_TILES; ++t) {
#ifdef DGS_PRODUCT_TILE      // (a CPU build that is to reach one kind on small matrices)
        if (t != ((DGS_PRODUCT_TILE == TILE_TALL || DGS_PRODUCT_TILE == TILE_192) && more != DGS_PRODUCT_TILE ? TILE_128 : DGS_PRODUCT_TILE)) continue;
#endif
        if ((t == TILE_TALL || t == TILE_192) && t != more) continue;
        const float us = tile_time(t, tiles(tile_high(t), tile_wide(t)), steps);
        if (least == 0.0f || us < least) {
            least = us;
            best = t;
        }
    }
    return best;
}

// How many splits of a sum of `steps` steps are tried: four steps each at least, `most` splits.  (A CPU build may ask for a number.)
static inline uint32_t splits_tried(uint32_t steps, uint32_t most)
{
#ifdef DGS_PRODUCT_SPLITS
    return steps < DGS_PRODUCT_SPLITS ? steps : DGS_PRODUCT_SPLITS;
#endif
    return steps / 4 > most ? most : steps / 4 < 1 ? 1u : steps / 4;
}
#ifdef DGS_PRODUCT_SPLITS
constexpr bool MOST_SPLITS = true;      // the last number that is tried
#else
constexpr bool MOST_SPLITS = false;     // the one with the least time
#endif

}  // namespace dgs
