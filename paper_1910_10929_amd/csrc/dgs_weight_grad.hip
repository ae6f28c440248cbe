// Gradient of a linear layer whose input is kept as a checkpoint: dw = dy^T values on the matrix units, summed over rows.
//
// A checkpoint's values are exact in bfloat16, so the codes become matrix operands without a second rounding; so does dy,
// in one part (bfloat16), two (half: 11 bits) or three (fp32: 24 bits), each taken off the rest by truncation.  Products
// are then exact in fp32 and only the sums round.  (The matrix units keep subnormal parts, whose unit is 2^-133: an fp32 value
// below 2^-110 loses what is less.)
//
// Both operands have the summed index (the row) outermost in memory.  They are staged in LDS as they lie, 16 bytes a lane,
// and turned on the way out by the transposing LDS read, four rows of 16 columns to 16 lanes.
//
// Bound by the matrix units where the product is large (32768 rows, 4096 x 4096, bfloat16: 953 to 1029 us from card to card,
// 1070 to 1150 TFLOP/s; a matrix product of the library's reaches 1260), by the partial sums of the split rows and by the tiles'
// first and last steps where it is not (8192 rows, 2304 x 768: 53 us a call, 550 TFLOP/s, of which the sums are 10 by themselves;
// 1500 rows, 1001 x 333, fp32: 24.7, the sums 5).
#include "dgs_rows.h"

namespace dgs {

constexpr uint32_t GRAD_TILE = 128;          // outputs and columns of a workgroup's tile
constexpr uint32_t GRAD_STEP = 32;           // rows staged at a time
constexpr uint32_t GRAD_THREADS = 256;  // four wavefronts, 64 x 64 of the tile each

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));      // eight bfloat16 of a lane
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

#ifdef DGS_HOST_EMULATION
}  // namespace dgs
#include "emu_matrix.h"
namespace dgs {
#else
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// c += a b: 32 x 32, 16 deep.  Lane l holds row (column) l % 32 of a (b), values 8 (l / 32) to 8 (l / 32) + 7 of the sum's
// index, and column l % 32 of c, rows (j % 4) + 8 (j / 4) + 4 (l / 32).
__device__ __forceinline__ f32x16 matrix_unit(u32x4 a, u32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Sixteen lanes read 8 bytes each, four 16-bit values of row j / 4 from column 4 (j % 4) on; lane j gets column j of the four rows.
__device__ __forceinline__ u32x2 read_turned(const uint16_t *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}
#endif

// The upper halves of two words, `lo`'s below.
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi)
{
#ifdef DGS_HOST_EMULATION
    return (lo >> 16) | (hi & 0xFFFF0000u);
#else
    return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
#endif
}

// A NaN with its mark in the upper half.
__device__ __forceinline__ float quiet(float v)
{
#ifdef DGS_HOST_EMULATION
    return v != v ? __uint_as_float(__float_as_uint(v) | 0x00400000u) : v;
#else
    return __builtin_canonicalizef(v);
#endif
}

// The parts of eight values, eight bfloat16 each.
template <class T> constexpr int PARTS = sizeof(T) == 4 ? 3 : __is_same(T, bf16) ? 1 : 2;

template <class T> __device__ __forceinline__ void split8(const Raw8<T> &r, u32x4 (&part)[PARTS<T>])
{
    if constexpr (PARTS<T> == 1) {
        __builtin_memcpy(&part[0], &r, sizeof(r));
    } else {
        float v[8];
        unpack8(r, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = quiet(v[i]);
#pragma unroll
        for (int p = 0; p < PARTS<T>; ++p) {
#pragma unroll
            for (int i = 0; i < 4; ++i) part[p][i] = upper_halves(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]));
            if (p + 1 == PARTS<T>) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float left = v[i] - __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u);
                // (of infinities and NaN, nothing; what is left of a number is one)
                v[i] = p > 0 || __builtin_isfinite(v[i]) ? left : 0.0f;
            }
        }
    }
}

// Eight codes as bfloat16.
__device__ __forceinline__ u32x4 values8(const uint32_t (&q)[2], uint32_t byte)
{
    float v[8];
    decode8(q, run_scale(byte), v);
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = upper_halves(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]));
    return o;
}

struct GradArgs {
    const void *dy;
    const int8_t *codes;
    const uint8_t *exps;
    const float *scale;
    float *dw, *sums, *bias_sums;       // where the tiles go: dw itself, or partial sums (splits x outs x cols); splits x col tiles x outs
    uint64_t dy_stride, codes_stride, exps_stride, dw_stride;
    uint32_t rows, outs, cols, split_rows, col_tiles, tiles, accumulate;
    // one split of few rows: every tile adds up its own rows of the bias gradient, and nothing is left to a second launch
    const float *shift;
    float *db;
    uint32_t own_bias;
};

// Where eight values of row k, columns 8 c to 8 c + 7, lie in a staged matrix: rows of GRAD_TILE values, their 16-byte pieces
// exchanged by row so that the four rows that 32 lanes read 64 bytes of are in different banks.
__device__ __forceinline__ uint32_t staged_at(uint32_t k, uint32_t c) { return k * GRAD_TILE + ((c ^ ((k & 3u) << 2)) << 3); }

// Any shape: every load looks at what is there.  For what the large tiles' loads take for granted and these matrices have not
// (fewer than 32 rows, fewer than eight outputs or columns); elsewhere it takes 2 to 2.5 times as long (32768 rows, 4096 x
// 4096: 2344 us; 8192 rows, 2304 x 768: 97).  20 rows, 4096 x 4096, bfloat16: 17.5 us, with the bias terms 21: 67 MB
// written at 3.8 and 3.2 TB/s, four bytes a lane, where a copy moves 5.0 to 5.4; 1 row, 8192 x 8192: 57 us, 4.7 TB/s.
template <class T>
__global__ __launch_bounds__(GRAD_THREADS) void k_weight_grad(GradArgs a)
{
    constexpr int P = PARTS<T>;
    constexpr uint32_t PER = GRAD_STEP * GRAD_TILE / 8 / GRAD_THREADS;      // pieces of eight a thread stages
    __shared__ __attribute__((aligned(16))) uint16_t la[2][P][GRAD_STEP * GRAD_TILE], lb[2][GRAD_STEP * GRAD_TILE];
    const uint32_t lane = lane_id(), wave = threadIdx.x >> 6;
    // neighbouring workgroups go to different dies: give each die a run of tiles of the same rows
    const uint32_t total = gridDim.x, die = blockIdx.x & 7u;
    const uint32_t at = (die * (total >> 3) + min(die, total & 7u)) + (blockIdx.x >> 3);
    const uint32_t split = at / a.tiles, tile = at - split * a.tiles;
    const uint32_t tile_o = tile / a.col_tiles, tile_c = tile - tile_o * a.col_tiles;
    const uint32_t row_first = split * a.split_rows;
    const uint32_t row_end = min(a.rows - row_first, a.split_rows) + row_first;
    const uint32_t steps = (row_end - row_first + GRAD_STEP - 1) / GRAD_STEP;

    // what this thread stages: piece threadIdx % 16 of rows threadIdx / 16 + 16 p
    const uint32_t piece = threadIdx.x & 15u, first_k = threadIdx.x >> 4;
    const uint32_t o0 = tile_o * GRAD_TILE + piece * 8, c0 = tile_c * GRAD_TILE + piece * 8;
    const uint32_t no = live8(o0, a.outs), nc = live8(c0, a.cols);
    Raw8<T> ra[PER];
    uint32_t rq[PER][2], rb[PER];
    auto fetch = [&](uint32_t step) {
#pragma unroll
        for (uint32_t p = 0; p < PER; ++p) {
            const uint32_t row = row_first + step * GRAD_STEP + first_k + 16 * p;
            const bool in = row < row_end;
            ra[p] = load8((const T *)a.dy + (in && no ? row * a.dy_stride + o0 : 0u), in ? no : 0u);
            load_codes(a.codes + (in && nc ? row * a.codes_stride + c0 : 0u), in ? nc : 0u, rq[p]);
            rb[p] = in && nc ? a.exps[row * a.exps_stride + c0 / DGS_CHECKPOINT_RUN] : 1u;
        }
    };
    auto stage = [&](uint32_t buf) {
#pragma unroll
        for (uint32_t p = 0; p < PER; ++p) {
            const uint32_t to = staged_at(first_k + 16 * p, piece);
            u32x4 part[P];
            split8(ra[p], part);
#pragma unroll
            for (int i = 0; i < P; ++i) *(u32x4 *)&la[buf][i][to] = part[i];
            *(u32x4 *)&lb[buf][to] = values8(rq[p], rb[p]);
        }
    };
    // the fragment of 32 columns from 8 c on, rows k to k + 15
    const uint32_t turn_k = ((lane >> 5) << 3) + ((lane & 15u) >> 2), turn_c = ((lane >> 4) & 1u) * 2u + ((lane & 3u) >> 1);
    auto fragment = [&](const uint16_t *m, uint32_t k, uint32_t c) {
        u32x4 f;
#pragma unroll
        for (uint32_t r = 0; r < 2; ++r) {
            const uint32_t row = k + turn_k + 4 * r;
            const u32x2 v = read_turned(m + staged_at(row, c + turn_c) + (lane & 1u) * 4);
            f[2 * r] = v.x;
            f[2 * r + 1] = v.y;
        }
        return f;
    };
    f32x16 acc[2][2], bias[2];
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[0][0][j] = acc[0][1][j] = acc[1][0][j] = acc[1][1][j] = bias[0][j] = bias[1][j] = 0.0f;
    const uint32_t wo = (wave >> 1) * 8, wc = (wave & 1u) * 8;      // this wavefront's corner, in pieces
    u32x4 ones;
#pragma unroll
    for (int i = 0; i < 4; ++i) ones[i] = 0x3F803F80u;

    if (steps) {
        fetch(0);
        stage(0);
    }
    __syncthreads();
    uint32_t bias_turn = 0;      // step % col_tiles: the column tiles share out the rows of the bias gradient
    for (uint32_t step = 0; step < steps; ++step) {
        const uint32_t buf = step & 1u;
        if (step + 1 < steps) fetch(step + 1);
        const bool bias_step = a.own_bias || (a.bias_sums && bias_turn == tile_c && wc == 0);
        bias_turn = bias_turn + 1 == a.col_tiles ? 0 : bias_turn + 1;
#pragma unroll
        for (uint32_t k = 0; k < GRAD_STEP; k += 16) {
            u32x4 fb[2];
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) fb[j] = fragment(lb[buf], k, wc + 4 * j);
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (uint32_t i = 0; i < 2; ++i) {
                    const u32x4 fa = fragment(la[buf][p], k, wo + 4 * i);
                    acc[i][0] = matrix_unit(fa, fb[0], acc[i][0]);
                    acc[i][1] = matrix_unit(fa, fb[1], acc[i][1]);
                    if (bias_step) bias[i] = matrix_unit(fa, ones, bias[i]);
                }
            }
        }
        if (step + 1 < steps) stage(buf ^ 1u);
        __syncthreads();
    }

    const bool whole = a.dw != nullptr;      // otherwise partial sums
    float *const out = whole ? a.dw : a.sums + (uint64_t)split * a.outs * a.cols;
    const uint64_t stride = whole ? a.dw_stride : a.cols;
    const uint32_t first_row = tile_o * GRAD_TILE + wo * 8 + 4 * (lane >> 5);
    const uint32_t there = a.outs - min(a.outs, first_row);      // rows from this lane's first on
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
        const uint32_t c = tile_c * GRAD_TILE + wc * 8 + 32 * j + (lane & 31u);
        if (c >= a.cols) continue;
        if (whole && a.scale) {
            const float scale = a.scale[c];
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) acc[i][j][r] *= scale;
        }
        if (a.own_bias && a.shift) {
            const float shift = a.shift[c];
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) acc[i][j][r] = __builtin_fmaf(bias[i][r], shift, acc[i][j][r]);
        }
        float *const to = out + (uint64_t)first_row * stride + c;
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
            for (uint32_t r = 0; r < 16; ++r) {
                const uint32_t o = 32 * i + (r & 3u) + 8 * (r >> 2);
                if (o >= there) continue;
                float *const p = to + o * stride;
                *p = whole && a.accumulate ? *p + acc[i][j][r] : acc[i][j][r];
            }
    }
    if (((a.own_bias && a.db && tile_c == 0) || a.bias_sums) && wc == 0 && (lane & 31u) == 0) {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
            for (uint32_t r = 0; r < 16; ++r) {
                const uint32_t o = tile_o * GRAD_TILE + wo * 8 + 32 * i + (r & 3u) + 8 * (r >> 2) + 4 * (lane >> 5);
                if (o >= a.outs) continue;
                if (a.own_bias) a.db[o] = a.accumulate ? a.db[o] + bias[i][r] : bias[i][r];
                else a.bias_sums[((uint64_t)split * a.col_tiles + tile_c) * a.outs + o] = bias[i][r];
            }
    }
}

// ---------------------------------------------------------------------------
// the large tiles
// ---------------------------------------------------------------------------
// 256 x 256 to eight wavefronts (128 x 64 each), 256 x 128 to eight and 128 x 128 to four (64 x 64 each).  Per 16 rows a
// wavefront of the first reads 6 KB of LDS for 8 matrix instructions, of the others 4 KB for 4 (of bfloat16; each further part
// of dy 4 KB for 8, and 2 KB for 4).  Two wavefronts to a SIMD do not hide the waits by themselves, so the overlap is written
// down: a step goes in units, one part of dy in a slice of 16 rows each; the fragments of a unit are read while the one before
// is multiplied, the next step's rows are staged between the units, the step after is asked for as soon as its registers
// are free, and the barrier stands before a step's last unit, behind which the first fragments of the next step are read.  A
// step is one basic block (the rows that fill no step come first, addresses are scalar, nothing looks at a bound), which
// the compiler can then order.
// At 32768 rows, 4096 x 4096, bfloat16: 256 x 256 with four wavefronts of 128 x 128 took 1047 us, with eight 982, with the order
// below 968; with branches around the loads 1680.  Half and fp32 take 2093 and 2595 us there, 3285 and 4075 on 256 x 128
// with all parts' fragments held at a time and three times the instructions to split a value.  At 8192 rows, 2304 x 768,
// bfloat16: 128 x 128 57 us, 256 x 128 53 (half the partial sums).
template <uint32_t WIDTH> __device__ __forceinline__ uint32_t wide_at(uint32_t k, uint32_t c) { return k * WIDTH + ((c ^ ((k & 3u) << 2)) << 3); }

template <uint32_t W> struct Width { static constexpr uint32_t value = W; };

// Between two matrix instructions: fragment reads, a share of what the next step's staging takes.  (Four vector instructions
// to one matrix instruction; with three or five 1040 and 1009 us in place of 968 at 32768 rows, 4096 x 4096.)
template <int COUNT> __device__ __forceinline__ void interleave(bool staging)
{
#ifndef DGS_HOST_EMULATION
    if (staging) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);      // matrix
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // LDS read
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);      // vector
            if (i % 3 == 0) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);      // LDS write
            if (i % 2 == 0) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);      // memory read
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
    }
#endif
}

template <class T, uint32_t STEP, uint32_t OUTS, uint32_t COLS, uint32_t WAVES, uint32_t TALL, bool RAGGED>
__global__ __launch_bounds__(WAVES * 64, 2) void k_weight_grad_tile(GradArgs a)
{
    constexpr int P = PARTS<T>;
    // wavefronts: TALL of them one below another, SIDE beside each other, I x J squares of 32 x 32 to each
    constexpr uint32_t THREADS = WAVES * 64, SIDE = WAVES / TALL, I = OUTS / 32 / TALL, J = COLS / 32 / SIDE, SLICES = STEP / 16;
    // staging: pieces of eight columns, rows from pass to pass, passes -- of dy, and of the codes
    constexpr uint32_t PIECES_O = OUTS / 8, APART_O = THREADS / PIECES_O, PASSES_O = STEP / APART_O;
    constexpr uint32_t PIECES_C = COLS / 8, APART_C = THREADS / PIECES_C, PASSES_C = STEP / APART_C;
    __shared__ __attribute__((aligned(16))) uint16_t la[2][P][STEP * OUTS], lb[2][STEP * COLS];
    const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6);
    const uint32_t total = gridDim.x, die = blockIdx.x & 7u;
    const uint32_t at = (die * (total >> 3) + min(die, total & 7u)) + (blockIdx.x >> 3);
    const uint32_t split = at / a.tiles, tile = at - split * a.tiles;
    const uint32_t tile_o = tile / a.col_tiles, tile_c = tile - tile_o * a.col_tiles;
    const uint32_t row_first = split * a.split_rows;
    const uint32_t row_end = min(a.rows - row_first, a.split_rows) + row_first;
    const uint32_t steps = (row_end - row_first + STEP - 1) / STEP;

    // what this thread stages
    const uint32_t piece_o = threadIdx.x % PIECES_O, first_o = threadIdx.x / PIECES_O;
    const uint32_t piece_c = threadIdx.x % PIECES_C, first_c = threadIdx.x / PIECES_C;
    const Place8 po = place8<false>(tile_o * OUTS + piece_o * 8, a.outs), pc = place8<false>(tile_c * COLS + piece_c * 8, a.cols);
    const uint32_t run = min(pc.c, a.cols - 1u) / DGS_CHECKPOINT_RUN;
    // (whether a row ends inside one of this tile's pieces)
    const bool cut_o = RAGGED && tile_o * OUTS + OUTS > a.outs, cut_c = RAGGED && tile_c * COLS + COLS > a.cols;
    Raw8<T> ra[PASSES_O];
    uint32_t rq[PASSES_C][2], rb[PASSES_C];
    // Step 0 holds the rows that do not fill a step, and the others are full: no step in the loop has to look.
    const uint32_t head = row_end - row_first - (steps - 1) * STEP;
    // In the loop addresses are scalar: pointers to a pass's first row, and an offset a lane.
    const uint64_t dy_bytes = a.dy_stride * sizeof(T);
    const uint32_t dy_lane = first_o * (uint32_t)dy_bytes + po.at * (uint32_t)sizeof(T);
    const uint32_t codes_lane = first_c * (uint32_t)a.codes_stride + pc.at, exps_lane = first_c * (uint32_t)a.exps_stride + run;
    const char *dy_p;
    const int8_t *codes_p;
    const uint8_t *exps_p;
    auto point_to = [&](uint32_t r) {
        dy_p = (const char *)a.dy + r * dy_bytes;
        codes_p = a.codes + r * a.codes_stride;
        exps_p = a.exps + r * a.exps_stride;
    };
    auto fetch_o = [&](uint32_t p) {
        const u32x4_any *const d = (const u32x4_any *)(dy_p + dy_lane);
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T) / 2; ++i) {
            const u32x4_any v = d[i];
            ra[p].w[4 * i] = v.x; ra[p].w[4 * i + 1] = v.y; ra[p].w[4 * i + 2] = v.z; ra[p].w[4 * i + 3] = v.w;
        }
        dy_p += APART_O * dy_bytes;
    };
    auto fetch_c = [&](uint32_t p) {
        const u32x2_any q = *(const u32x2_any *)(codes_p + codes_lane);
        rq[p][0] = q.x;
        rq[p][1] = q.y;
        rb[p] = exps_p[exps_lane];
        codes_p += APART_C * a.codes_stride;
        exps_p += APART_C * a.exps_stride;
    };
    float bias[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) bias[i] = 0.0f;
    uint32_t bias_turn = 0;     // step % col_tiles: the column tiles share out the rows of the bias gradient
    auto add_bias = [&](uint32_t there) {
        if (a.own_bias || (a.bias_sums && bias_turn == tile_c)) {
#pragma unroll
            for (uint32_t p = 0; p < PASSES_O; ++p) {
                if (first_o + APART_O * p >= there) continue;
                Raw8<T> r = ra[p];
                if (cut_o) in_place<false>(r, po);
                float v[8];
                unpack8(r, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) bias[i] += v[i];
            }
        }
        bias_turn = bias_turn + 1 == a.col_tiles ? 0 : bias_turn + 1;
    };
    auto stage_o = [&](uint32_t buf, uint32_t p) {
        if (cut_o) in_place<false>(ra[p], po);
        const uint32_t to = wide_at<OUTS>(first_o + APART_O * p, piece_o);
        u32x4 part[P];
        split8(ra[p], part);
#pragma unroll
        for (int i = 0; i < P; ++i) *(u32x4 *)&la[buf][i][to] = part[i];
    };
    auto stage_c = [&](uint32_t buf, uint32_t p) {
        if (cut_c) codes_in_place<false>(rq[p], pc);
        *(u32x4 *)&lb[buf][wide_at<COLS>(first_c + APART_C * p, piece_c)] = values8(rq[p], rb[p]);
    };
    const uint32_t turn_k = ((lane >> 5) << 3) + ((lane & 15u) >> 2), turn_c = ((lane >> 4) & 1u) * 2u + ((lane & 3u) >> 1);
    auto fragment = [&](const uint16_t *m, auto width, uint32_t k, uint32_t c) {
        u32x4 f;
#pragma unroll
        for (uint32_t r = 0; r < 2; ++r) {
            const u32x2 v = read_turned(m + wide_at<width.value>(k + turn_k + 4 * r, c + turn_c) + (lane & 1u) * 4);
            f[2 * r] = v.x;
            f[2 * r + 1] = v.y;
        }
        return f;
    };
    f32x16 acc[I][J];
#pragma unroll
    for (uint32_t i = 0; i < I; ++i)
#pragma unroll
        for (uint32_t j = 0; j < J; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    const uint32_t wo = wave / SIDE * (4 * I), wc = wave % SIDE * (4 * J);      // this wavefront's corner, in pieces
    // A step is multiplied in units, one part of dy in a slice of 16 rows each: fragments of the unit at hand and of the next.
    constexpr uint32_t UNITS = SLICES * P;
    u32x4 fa[2][I], fb[2][J];
    auto read = [&](uint32_t buf, uint32_t unit) {      // (sets by turns: UNITS and SLICES are even)
        const uint32_t slice = unit / P, part = unit % P;
        if (part == 0) {
#pragma unroll
            for (uint32_t j = 0; j < J; ++j) fb[slice & 1u][j] = fragment(lb[buf], Width<COLS>(), slice * 16, wc + 4 * j);
        }
#pragma unroll
        for (uint32_t i = 0; i < I; ++i) fa[unit & 1u][i] = fragment(la[buf][part], Width<OUTS>(), slice * 16, wo + 4 * i);
    };
    auto multiply = [&](uint32_t unit) {
#pragma unroll
        for (uint32_t i = 0; i < I; ++i)
#pragma unroll
            for (uint32_t j = 0; j < J; ++j) acc[i][j] = matrix_unit(fa[unit & 1u][i], fb[unit / P & 1u][j], acc[i][j]);
    };

#pragma unroll
    for (uint32_t p = 0; p < PASSES_O; ++p)      // (rows that are not there: the last one)
        ra[p] = load_at<false>((const T *)a.dy + min(row_first + first_o + APART_O * p, row_end - 1u) * a.dy_stride, po.at, a.outs);
#pragma unroll
    for (uint32_t p = 0; p < PASSES_C; ++p) {
        const uint32_t r = min(row_first + first_c + APART_C * p, row_end - 1u);
        load_codes_at<false>(a.codes + r * a.codes_stride, pc.at, a.cols, rq[p]);
        rb[p] = (a.exps + r * a.exps_stride)[run];
    }
    add_bias(head);
#pragma unroll
    for (uint32_t p = 0; p < PASSES_O; ++p) {
        if (first_o + APART_O * p >= head) {
#pragma unroll
            for (uint32_t i = 0; i < 2 * sizeof(T); ++i) ra[p].w[i] = 0;
        }
        stage_o(0, p);
    }
#pragma unroll
    for (uint32_t p = 0; p < PASSES_C; ++p) {
        if (first_c + APART_C * p >= head) {
            rq[p][0] = rq[p][1] = 0;
            rb[p] = 1;
        }
        stage_c(0, p);
    }
    // (what is asked for beyond the last step is not used: the matrix's last rows, of which there are enough)
    uint32_t row = row_first + head;
    point_to(min(row, a.rows - STEP));
#pragma unroll
    for (uint32_t p = 0; p < PASSES_O; ++p) fetch_o(p);
#pragma unroll
    for (uint32_t p = 0; p < PASSES_C; ++p) fetch_c(p);
    __syncthreads();
    read(0, 0);
    for (uint32_t step = 0; step < steps; ++step) {
        const uint32_t buf = step & 1u;
        add_bias(step + 1 < steps ? STEP : 0u);
        row += STEP;
        if (row > a.rows - STEP) point_to(a.rows - STEP);
#pragma unroll
        for (uint32_t unit = 0; unit < UNITS; ++unit) {
            if (unit + 1 < UNITS) {
                read(buf, unit + 1);
#pragma unroll
                for (uint32_t p = unit * PASSES_O / (UNITS - 1); p < (unit + 1) * PASSES_O / (UNITS - 1); ++p) {
                    constexpr uint32_t EACH = PASSES_O / PASSES_C;
                    stage_o(buf ^ 1u, p);
                    if (p % EACH == 0) stage_c(buf ^ 1u, p / EACH);
                    fetch_o(p);
                    if (p % EACH == 0) fetch_c(p / EACH);
                }
            } else {
                __syncthreads();
                read(buf ^ 1u, 0);
            }
            multiply(unit);
            interleave<2 * I * J>(unit + 1 < UNITS);
        }
    }

    // the bias gradient of this tile's rows: the threads of a piece of columns, one after another
    float *const sums = (float *)&la[0][0][0];
    if (a.bias_sums || a.own_bias) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[first_o * OUTS + piece_o * 8 + i] = bias[i];
        __syncthreads();
        const uint32_t o = tile_o * OUTS + threadIdx.x;
        float sum = 0.0f;
        if (threadIdx.x < OUTS) {
#pragma unroll
            for (uint32_t q = 0; q < APART_O; ++q) sum += sums[q * OUTS + threadIdx.x];
            if (o < a.outs && a.bias_sums) a.bias_sums[((uint64_t)split * a.col_tiles + tile_c) * a.outs + o] = sum;
            if (o < a.outs && a.own_bias && a.db && tile_c == 0) a.db[o] = a.accumulate ? a.db[o] + sum : sum;
        }
        if (a.own_bias) {
            __syncthreads();
            if (threadIdx.x < OUTS) sums[threadIdx.x] = sum;
            __syncthreads();
        }
    }
    const bool whole = a.dw != nullptr;      // otherwise partial sums
    float *const out = whole ? a.dw : a.sums + (uint64_t)split * a.outs * a.cols;
    const uint64_t stride = whole ? a.dw_stride : a.cols;
    const uint32_t first_row = wo * 8 + 4 * (lane >> 5);      // of the tile; this lane's rows are 32 i + (r % 4) + 8 (r / 4) behind it
#pragma unroll
    for (uint32_t j = 0; j < J; ++j) {
        const uint32_t c = tile_c * COLS + wc * 8 + 32 * j + (lane & 31u);
        if (c >= a.cols) continue;
        if (whole && a.scale) {
            const float scale = a.scale[c];
#pragma unroll
            for (uint32_t i = 0; i < I; ++i)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) acc[i][j][r] *= scale;
        }
        if (a.own_bias && a.shift) {
            const float shift = a.shift[c];
#pragma unroll
            for (uint32_t i = 0; i < I; ++i)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r)
                    acc[i][j][r] = __builtin_fmaf(sums[first_row + 32 * i + (r & 3u) + 8 * (r >> 2)], shift, acc[i][j][r]);
        }
        float *const to = out + (uint64_t)(tile_o * OUTS + first_row) * stride + c;
        const uint32_t there = a.outs - min(a.outs, tile_o * OUTS + first_row);      // rows from this lane's first on
#pragma unroll
        for (uint32_t i = 0; i < I; ++i)
#pragma unroll
            for (uint32_t r = 0; r < 16; ++r) {
                const uint32_t o = 32 * i + (r & 3u) + 8 * (r >> 2);
                if (o >= there) continue;
                float *const p = to + o * stride;
                *p = whole && a.accumulate ? *p + acc[i][j][r] : acc[i][j][r];
            }
    }
}

// Adds up the splits' partial sums (where there are any) and finishes: a wavefront an output row and 256 columns, four to a lane.
// Bound by the latency of few loads: 2304 x 768 in four splits, 35 MB from cache and memory, 10 us (6.8 without bias terms);
// 1001 x 333 5 us.  A wavefront takes its splits eight at a time, one after another: 64 x 64 in 512 splits 57 us, 128 x 128 25.
__global__ __launch_bounds__(256) void k_weight_grad_finish(const float *sums, const float *bias_sums, const float *scale,
                                                            const float *shift, float *dw, uint64_t dw_stride, float *db, uint32_t outs,
                                                            uint32_t cols, uint32_t splits, uint32_t bias_parts, uint32_t accumulate)
{
    const uint32_t o = blockIdx.x * 4 + uniform(threadIdx.x >> 6), c = blockIdx.y * 256 + lane_id() * 4;
    if (o >= outs) return;
    const uint32_t n = !dw || c >= cols ? 0u : min(4u, cols - c);
    float bias = 0.0f, s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (bias_sums) {
        for (uint32_t p = lane_id(); p < bias_parts; p += 64) bias += bias_sums[(uint64_t)p * outs + o];
    }
    if (n && cols >= 4) {
        // (four that exist, eight splits' at a time: where a row ends inside a lane's four, those before its end)
        const uint32_t at = min(c, cols - 4u);
        const float *const p = sums + (uint64_t)o * cols + at;
        for (uint32_t i = 0; i < splits; i += 8) {
            f32x4_any v[8];
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[j] = *(const f32x4_any *)(p + (uint64_t)min(i + j, splits - 1u) * outs * cols);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                if (i + j >= splits) continue;
                s[0] += v[j].x; s[1] += v[j].y; s[2] += v[j].z; s[3] += v[j].w;
            }
        }
        if (c != at) {
            const uint32_t by = c - at;
            s[0] = by == 1 ? s[1] : by == 2 ? s[2] : s[3];
            s[1] = by == 1 ? s[2] : s[3];
            s[2] = s[3];
        }
    } else {
        for (uint32_t i = 0; i < splits; ++i)
            for (uint32_t j = 0; j < n; ++j) s[j] += sums[((uint64_t)i * outs + o) * cols + c + j];
    }
    if (bias_sums) {
        bias = wave_sum(bias);
        if (db && blockIdx.y == 0 && lane_id() == 0) db[o] = accumulate ? db[o] + bias : bias;
    }
    if (n == 0) return;
    float *const q = dw + o * dw_stride + c;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        if (j >= n) continue;
        if (scale) s[j] *= scale[c + j];
        if (shift) s[j] = __builtin_fmaf(bias, shift[c + j], s[j]);
        if (accumulate) s[j] += q[j];
    }
    if (n == 4) {
        f32x4_any v;
        v.x = s[0]; v.y = s[1]; v.z = s[2]; v.w = s[3];
        *(f32x4_any *)q = v;
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (j < n) q[j] = s[j];
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

// The tiles, largest first, and how a workgroup of each was timed: microseconds for a step of 64 rows with every compute unit
// busy, for what comes before and behind the steps, and workgroups that run at a time.
struct GradTile {
    uint32_t outs, cols, step, at_once;
    float per_step, fixed;
};
enum { TILE_256, TILE_256_128, TILE_128, TILE_ANY, TILES };
static GradTile tile_of(int tile, int type)
{
    const int i = type == DGS_BF16 ? 0 : type == DGS_F16 ? 1 : 2;
    constexpr float us_256[3] = {1.94f, 4.08f, 5.06f}, us_256_128[3] = {1.22f, 2.37f, 3.21f}, us_128[3] = {1.46f, 2.67f, 3.46f},
                    us_any[3] = {3.0f, 5.0f, 7.0f};
    switch (tile) {
    case TILE_256: return GradTile{256, 256, i == 0 ? 64u : 32u, 256, us_256[i], 8.0f};
    case TILE_256_128: return GradTile{256, 128, i == 0 ? 64u : 32u, 256, us_256_128[i], 11.0f};
    case TILE_128: return GradTile{128, 128, 32, 512, us_128[i], 7.0f};
    default: return GradTile{GRAD_TILE, GRAD_TILE, GRAD_STEP, 512, us_any[i], 7.0f};
    }
}

struct GradPlan {
    int tile;
    uint32_t out_tiles, col_tiles, splits, split_rows;
};
static GradPlan plan_of(int tile, uint32_t rows, uint32_t outs, uint32_t cols, int type, bool one_split, float &us)
{
    const GradTile t = tile_of(tile, type);
    GradPlan g;
    g.tile = tile;
    g.out_tiles = (outs - 1) / t.outs + 1;
    g.col_tiles = (cols - 1) / t.cols + 1;
    const uint64_t tiles = (uint64_t)g.out_tiles * g.col_tiles;
    const uint32_t steps = rows ? (rows - 1) / t.step + 1 : 0;
    uint64_t splits = tiles >= t.at_once || one_split ? 1 : t.at_once / tiles;
    if (splits > steps / 4) splits = steps / 4;      // at least four steps each
    if (splits < 1) splits = 1;
    g.split_rows = (steps + (uint32_t)splits - 1) / (uint32_t)splits * t.step;
    g.splits = g.split_rows ? (rows - 1) / g.split_rows + 1 : 1;
    const float rounds = (float)((tiles * g.splits - 1) / t.at_once + 1);
    us = rounds * ((float)g.split_rows / 64.0f * t.per_step + t.fixed);
    if (g.splits > 1) us += 4.0f + (float)g.splits * (float)outs * (float)cols * 8.0f / 4.5e6f;      // partial sums there and back
    return g;
}
// The tile and the number of splits that should take the least time.  (20 rows of 4096 x 4096 took 80 us in partial sums and
// take 21 in one launch; 8192 rows of 2304 x 768 are 54 tiles, which without splits would leave 202 compute units idle.)  What
// a whole tile's loads take for granted -- a step's rows, eight columns -- the last kind does without.
static GradPlan grad_plan(uint32_t rows, uint32_t outs, uint32_t cols, int type)
{
    const bool any = rows < 32 || outs < 8 || cols < 8;
    GradPlan g = {};
    float best = 0.0f;
    for (int tile = any ? TILE_ANY : TILE_256; tile <= (any ? TILE_ANY : TILE_128); ++tile) {
        if (rows < tile_of(tile, type).step && !any) continue;
#ifdef DGS_GRAD_TILE      // (a CPU build that is to reach one kind on small matrices)
        if (!any && tile != DGS_GRAD_TILE) continue;
#endif
        for (int one = 0; one < 2; ++one) {
            float us;
            const GradPlan other = plan_of(tile, rows, outs, cols, type, one != 0, us);
            if (best == 0.0f || us < best) {
                best = us;
                g = other;
            }
        }
    }
    return g;
}
template <class T, uint32_t STEP, uint32_t OUTS, uint32_t COLS, uint32_t WAVES, uint32_t TALL>
static void launch_tile(const GradArgs &a, dim3 grid, hipStream_t st)
{
    if ((a.outs | a.cols) & 7u) hipLaunchKernelGGL((k_weight_grad_tile<T, STEP, OUTS, COLS, WAVES, TALL, true>), grid, dim3(WAVES * 64), 0, st, a);
    else hipLaunchKernelGGL((k_weight_grad_tile<T, STEP, OUTS, COLS, WAVES, TALL, false>), grid, dim3(WAVES * 64), 0, st, a);
}
template <class T> static void launch_grad(const GradArgs &a, int tile, dim3 grid, hipStream_t st)
{
    constexpr uint32_t STEP = PARTS<T> == 1 ? 64 : 32;
    if (tile == TILE_256) launch_tile<T, STEP, 256, 256, 8, 2>(a, grid, st);
    else if (tile == TILE_256_128) launch_tile<T, STEP, 256, 128, 8, 4>(a, grid, st);
    else if (tile == TILE_128) launch_tile<T, 32, 128, 128, 4, 2>(a, grid, st);
    else hipLaunchKernelGGL(k_weight_grad<T>, grid, dim3(GRAD_THREADS), 0, st, a);
}
// floats of partial sums, and of bias sums
static void grad_sizes(const GradPlan &g, uint32_t outs, uint32_t cols, uint64_t &sums, uint64_t &bias)
{
    sums = (uint64_t)g.splits * outs * cols;
    bias = (uint64_t)g.splits * g.col_tiles * outs;
}

}  // namespace dgs

using namespace dgs;

extern "C" size_t dgs_checkpoint_weight_grad_workspace(uint32_t rows, uint32_t outs, uint32_t cols, int type)
{
    if (outs == 0 || cols == 0 || !is_type(type)) return 0;
    uint64_t sums, bias;
    grad_sizes(grad_plan(rows, outs, cols, type), outs, cols, sums, bias);
    return (size_t)(sums + bias) * sizeof(float);
}

extern "C" int dgs_checkpoint_weight_grad(const dgs_weight_grad_args *args, void *hip_stream)
{
    if (!args) return DGS_EINVAL;
    const dgs_weight_grad_args &p = *args;
    if (p.outs == 0 || p.cols == 0 || !is_type(p.type)) return DGS_EINVAL;
    if (!matrix_ok(p.dw, p.dw_stride, p.cols, DGS_F32) || !aligned_to(p.scale, 4) || !aligned_to(p.shift, 4) || !aligned_to(p.db, 4))
        return DGS_EINVAL;
    if (p.rows && (!matrix_ok(p.dy.data, p.dy.stride, p.outs, p.type) || !codes_ok(p.saved, p.cols))) return DGS_EINVAL;
    const GradPlan g = grad_plan(p.rows, p.outs, p.cols, p.type);
    const uint64_t blocks = (uint64_t)g.out_tiles * g.col_tiles * g.splits;
    // (a lane's offset, at most 31 rows, is held in 32 bits)
    if (p.dy.stride * type_bytes(p.type) >= (1u << 27) || p.saved.codes_stride >= (1u << 27) || p.saved.exps_stride >= (1u << 27)) return DGS_ENOTSUP;
    if (p.rows > 0x7FFFFFFFu || p.outs > 0x7FFFFFu || p.cols > 0x7FFFFFu || blocks > 0xFFFFFFu) return DGS_ENOTSUP;
    uint64_t sums, bias;
    grad_sizes(g, p.outs, p.cols, sums, bias);
    if (!p.workspace || !aligned_to(p.workspace, 16)) return DGS_EINVAL;
    if (p.workspace_bytes < (sums + bias) * sizeof(float)) return DGS_ENOMEM;
    const hipStream_t st = (hipStream_t)hip_stream;
    // (beyond a few rows, tiles that all add up the same rows cost more than the second launch)
    const bool own_bias = g.splits == 1 && p.rows <= 256 && (p.db || p.shift);
    const bool partial = g.splits > 1 || (p.shift && !own_bias);
    GradArgs a;
    a.dy = p.dy.data; a.codes = p.saved.codes; a.exps = p.saved.exps;
    a.scale = p.scale;
    a.dw = partial ? nullptr : p.dw;
    a.sums = (float *)p.workspace;
    a.bias_sums = (p.db || p.shift) && !own_bias ? a.sums + sums : nullptr;
    a.shift = p.shift;
    a.db = p.db;
    a.own_bias = own_bias;
    a.dy_stride = p.dy.stride; a.codes_stride = p.saved.codes_stride; a.exps_stride = p.saved.exps_stride; a.dw_stride = p.dw_stride;
    a.rows = p.rows; a.outs = p.outs; a.cols = p.cols;
    a.split_rows = g.split_rows;
    a.col_tiles = g.col_tiles; a.tiles = g.out_tiles * g.col_tiles;
    a.accumulate = p.accumulate != 0;
    const dim3 grid((uint32_t)blocks);
    if (p.type == DGS_F32) launch_grad<float>(a, g.tile, grid, st);
    else if (p.type == DGS_F16) launch_grad<f16>(a, g.tile, grid, st);
    else launch_grad<bf16>(a, g.tile, grid, st);
    if (partial || a.bias_sums)
        hipLaunchKernelGGL(k_weight_grad_finish, dim3((p.outs + 3) / 4, partial ? (p.cols + 255) / 256 : 1), dim3(256), 0, st,
                           (const float *)a.sums, (const float *)a.bias_sums, p.scale, p.shift, partial ? p.dw : nullptr, p.dw_stride,
                           p.db, p.outs, p.cols, g.splits, g.splits * g.col_tiles, a.accumulate);
    return launched();
}
