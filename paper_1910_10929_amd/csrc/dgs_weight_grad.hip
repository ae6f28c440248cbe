// Gradient of a linear layer whose input is kept as a checkpoint: dw = dy^T values on the matrix units, summed over rows.
//
// A checkpoint's values are exact in bfloat16, so the codes become matrix operands without a second rounding; so does dy,
// in one part (bfloat16), two (half: 11 bits) or three (fp32: 24 bits), each taken off the rest by truncation.  Products
// are then exact in fp32 and only the sums round.
//
// Both operands have the summed index (the row) outermost in memory.  They are staged in LDS as they lie, 16 bytes a lane,
// and turned on the way out by the transposing LDS read, four rows of 16 columns to 16 lanes.
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
        for (int p = 0; p < PARTS<T>; ++p) {
            uint32_t b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                b[i] = __float_as_uint(v[i]);
                // what is left; of infinities and NaN, nothing (a NaN may hold its mark in the low half)
                const bool finite = (b[i] & 0x7F800000u) != 0x7F800000u;
                if (!finite && (b[i] & 0x007FFFFFu)) b[i] |= 0x00400000u;
                v[i] = finite ? v[i] - __uint_as_float(b[i] & 0xFFFF0000u) : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) part[p][i] = (b[2 * i] >> 16) | (b[2 * i + 1] & 0xFFFF0000u);
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
    for (int i = 0; i < 4; ++i) o[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xFFFF0000u);
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
};

// Where eight values of row k, columns 8 c to 8 c + 7, lie in a staged matrix: rows of GRAD_TILE values, their 16-byte pieces
// exchanged by row so that the four rows that 32 lanes read 64 bytes of are in different banks.
__device__ __forceinline__ uint32_t staged_at(uint32_t k, uint32_t c) { return k * GRAD_TILE + ((c ^ ((k & 3u) << 2)) << 3); }

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
        const bool bias_step = a.bias_sums && bias_turn == tile_c && wc == 0;
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
#pragma unroll
    for (uint32_t j = 0; j < 2; ++j) {
        const uint32_t c = tile_c * GRAD_TILE + wc * 8 + 32 * j + (lane & 31u);
        if (c >= a.cols) continue;
        const float scale = whole && a.scale ? a.scale[c] : 1.0f;
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
            for (uint32_t r = 0; r < 16; ++r) {
                const uint32_t o = tile_o * GRAD_TILE + wo * 8 + 32 * i + (r & 3u) + 8 * (r >> 2) + 4 * (lane >> 5);
                if (o >= a.outs) continue;
                float *p = out + o * stride + c;
                const float v = acc[i][j][r] * scale;
                *p = whole && a.accumulate ? *p + v : v;
            }
    }
    if (a.bias_sums && wc == 0 && (lane & 31u) == 0) {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
            for (uint32_t r = 0; r < 16; ++r) {
                const uint32_t o = tile_o * GRAD_TILE + wo * 8 + 32 * i + (r & 3u) + 8 * (r >> 2) + 4 * (lane >> 5);
                if (o < a.outs) a.bias_sums[((uint64_t)split * a.col_tiles + tile_c) * a.outs + o] = bias[i][r];
            }
    }
}

// Adds up the splits' partial sums (where there are any) and finishes: one output row a workgroup row, 256 columns a block.
__global__ __launch_bounds__(256) void k_weight_grad_finish(const float *sums, const float *bias_sums, const float *scale,
                                                            const float *shift, float *dw, uint64_t dw_stride, float *db, uint32_t outs,
                                                            uint32_t cols, uint32_t splits, uint32_t bias_parts, uint32_t accumulate)
{
    const uint32_t o = blockIdx.x, c = blockIdx.y * 256 + threadIdx.x;
    float bias = 0.0f;
    if (bias_sums) {
        for (uint32_t p = lane_id(); p < bias_parts; p += 64) bias += bias_sums[(uint64_t)p * outs + o];
        bias = wave_sum(bias);
        if (db && blockIdx.y == 0 && threadIdx.x == 0) db[o] = accumulate ? db[o] + bias : bias;
    }
    if (!dw || c >= cols) return;
    const float *p = sums + (uint64_t)o * cols + c;
    float s = 0.0f;
#pragma unroll 8
    for (uint32_t i = 0; i < splits; ++i) s += p[(uint64_t)i * outs * cols];
    if (scale) s *= scale[c];
    if (shift) s = __builtin_fmaf(bias, shift[c], s);
    float *q = dw + o * dw_stride + c;
    *q = accumulate ? *q + s : s;
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

struct GradPlan {
    uint32_t out_tiles, col_tiles, splits, split_rows;
};
static GradPlan grad_plan(uint32_t rows, uint32_t outs, uint32_t cols)
{
    GradPlan g;
    g.out_tiles = (outs - 1) / GRAD_TILE + 1;
    g.col_tiles = (cols - 1) / GRAD_TILE + 1;
    const uint64_t tiles = (uint64_t)g.out_tiles * g.col_tiles;
    const uint32_t steps = rows ? (rows - 1) / GRAD_STEP + 1 : 0;
    uint64_t splits = tiles >= 512 ? 1 : 512 / tiles;
    if (splits > steps / 4) splits = steps / 4;      // at least four steps each
    if (splits < 1) splits = 1;
    g.split_rows = (steps + (uint32_t)splits - 1) / (uint32_t)splits * GRAD_STEP;
    g.splits = g.split_rows ? (rows - 1) / g.split_rows + 1 : 1;
    return g;
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
    grad_sizes(grad_plan(rows, outs, cols), outs, cols, sums, bias);
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
    const GradPlan g = grad_plan(p.rows, p.outs, p.cols);
    const uint64_t blocks = (uint64_t)g.out_tiles * g.col_tiles * g.splits;
    if (p.rows > 0x7FFFFFFFu || p.outs > 0x7FFFFFu || p.cols > 0x7FFFFFu || blocks > 0xFFFFFFu) return DGS_ENOTSUP;
    uint64_t sums, bias;
    grad_sizes(g, p.outs, p.cols, sums, bias);
    if (!p.workspace || !aligned_to(p.workspace, 16)) return DGS_EINVAL;
    if (p.workspace_bytes < (sums + bias) * sizeof(float)) return DGS_ENOMEM;
    const hipStream_t st = (hipStream_t)hip_stream;
    const bool partial = g.splits > 1 || p.shift;
    GradArgs a;
    a.dy = p.dy.data; a.codes = p.saved.codes; a.exps = p.saved.exps;
    a.scale = p.scale;
    a.dw = partial ? nullptr : p.dw;
    a.sums = (float *)p.workspace;
    a.bias_sums = p.db || p.shift ? a.sums + sums : nullptr;
    a.dy_stride = p.dy.stride; a.codes_stride = p.saved.codes_stride; a.exps_stride = p.saved.exps_stride; a.dw_stride = p.dw_stride;
    a.rows = p.rows; a.outs = p.outs; a.cols = p.cols;
    a.split_rows = g.split_rows;
    a.col_tiles = g.col_tiles; a.tiles = g.out_tiles * g.col_tiles;
    a.accumulate = p.accumulate != 0;
    const dim3 grid((uint32_t)blocks), block(GRAD_THREADS);
    if (p.type == DGS_F32) hipLaunchKernelGGL(k_weight_grad<float>, grid, block, 0, st, a);
    else if (p.type == DGS_F16) hipLaunchKernelGGL(k_weight_grad<f16>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(k_weight_grad<bf16>, grid, block, 0, st, a);
    if (partial || p.db)
        hipLaunchKernelGGL(k_weight_grad_finish, dim3(p.outs, partial ? (p.cols + 255) / 256 : 1), dim3(256), 0, st,
                           (const float *)a.sums, (const float *)a.bias_sums, p.scale, p.shift, partial ? p.dw : nullptr, p.dw_stride,
                           p.db, p.outs, p.cols, g.splits, g.splits * g.col_tiles, a.accumulate);
    return launched();
}
