// The output layer with its loss: logits = x W^T + b, softmax cross entropy against one target a row, and the gradients, of
// which no logits are kept.
//
// Forward: a tile of logits stays in a workgroup's sums, of which each row's maximum and sum of exponentials go out; a second
// launch joins the tiles of a row.  Backward: the same tiles again, a piece of the vocabulary at a time; with the row's lse they
// become the gradient of the logits, which is written in 16-bit parts (HeadRow), and two products take dx and dweight from it.
//
// Numbers.  Sums, statistics and exponentials are fp32.  Logits are products of the operands as they are (bfloat16, half;
// fp32 in two halves, 22 bits, every row of x and of W scaled by a power of two of its own).  The gradient of the logits is divided by a power of two for each row (at least the larger
// of the incoming gradients) and held in two halves, the second times 2^11: 22 bits of a value down to 2^-28 of that power, below it steps
// of 2^-49 (11 bits of what a softmax of 2^-38 leaves; with the second half as it is 2^-38 would be the step).  dx in bfloat16 takes
// the first half, 11 bits where the result is rounded to 8, everything else both.  The other operand of these products is W or x in half,
// scaled by powers of two so that the largest magnitude lies below 2^15: a bfloat16 value is exact there down to 2^-31 of the
// largest, and what is lost of smaller ones is below 2^-39 of it (fp32, in two halves: 2^-50).  x carries the rows' powers of two.
#include "dgs_product.h"

namespace dgs {

// ---------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------

#ifdef DGS_HOST_EMULATION
constexpr uint32_t RANGE_BLOCKS = 256;
#else
constexpr uint32_t RANGE_BLOCKS = 1024;      // of rows, and as many of W
#endif
constexpr int NO_RANGE = -100000;           // nothing but zeros
constexpr int TOP = 15;                     // the largest magnitude of a scaled operand lies below 2^TOP
constexpr int GRAD_TOP = 14;                // a row's logit gradients are at most 2 after division
constexpr uint32_t LOW = 11;                // second halves are held times 2^LOW

// What a row of the backward pass needs: dlogit = pull * softmax - push * onehot, divided by 2^power and scaled to GRAD_TOP.
struct HeadRow {
    float lse, pull, push;
    int power;      // of the incoming gradients' larger one
};
// (such a row leaves no gradient, whatever it holds)
__device__ __forceinline__ bool nothing_arrives(const HeadRow &h) { return h.pull == 0.0f && h.push == 0.0f; }
struct Ranges {
    int *x, *w;         // one for each workgroup: largest exponent of x (with the rows' powers), of W
    int *w_least;       // ... and the smallest of a row of W that is not zeros
    int *row, *entry;   // of each row of x, of W
};
// Exponents by which the whole of x (with the rows' powers) and of W are multiplied in the gradients' products.  even: no row of an fp32 W
// lies so far below the largest that logits would miss its own power.
struct Scales { int x, w, even; };
// Logits of an fp32 W whose rows' largest values lie within 2^SPREAD take the copy that dx takes too: 22 bits of a value down to 2^-20 of
// its row's largest then, steps of 2^-41 below.  (432 x 3920 x 59264 with dx: one copy 1884 us, two 2075.)
constexpr int SPREAD = 8;

__device__ __forceinline__ int exponent_of(uint32_t magnitude)      // smallest e with |v| < 2^e
{
    return magnitude == 0 ? NO_RANGE : max((int)(magnitude >> 23), 1) - 126;
}
__device__ __forceinline__ int scale_of(int exponent) { return exponent <= NO_RANGE / 2 ? 0 : TOP - exponent; }
__device__ __forceinline__ float times_power(float v, int e)
{
#ifdef DGS_HOST_EMULATION
    return ldexpf(v, e);
#else
    return __builtin_amdgcn_ldexpf(v, e);
#endif
}
__device__ __forceinline__ float power_of_e(float v)      // e^v
{
#ifdef DGS_HOST_EMULATION
    return exp2f(v * 1.44269504f);
#else
    return __builtin_amdgcn_exp2f(v * 1.44269504f);
#endif
}
__device__ __forceinline__ float other_half(float v)      // the value of lane l ^ 32
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute((int)((lane_id() ^ 32u) << 2), (int)__float_as_uint(v)));
}
__device__ __forceinline__ int wave_max(int v)
{
#pragma unroll
    for (uint32_t by = 32; by; by >>= 1) v = max(v, __builtin_amdgcn_ds_bpermute((int)((lane_id() ^ by) << 2), v));
    return v;
}

struct Targets {
    const void *at;
    uint32_t wide;      // 64 bits each
    uint32_t vocab;
};
// A row's target, or the vocabulary's size where it is none of its entries.
__device__ __forceinline__ uint32_t target_of(const Targets &t, uint32_t row)
{
    if (t.wide) {
        const uint64_t v = ((const uint64_t *)t.at)[row];
        return v < t.vocab ? (uint32_t)v : t.vocab;
    }
    return min(((const uint32_t *)t.at)[row], t.vocab);
}

// Exponents of x, row by row, and of W; in a backward pass what the rows need besides.  A wavefront a row.  Bound by memory: x of
// 8192 x 4096 and W of 32768 x 4096 in bfloat16, 336 MB, 57 us (5.9 TB/s, part of it from cache).
template <class T>
__global__ __launch_bounds__(256) void k_head_range(const T *x, uint64_t x_stride, const T *w, uint64_t w_stride, uint32_t rows,
                                                    uint32_t cols, Targets targets, const float *lse, const float *dloss,
                                                    const float *dlse, HeadRow *row_info, Ranges to)
{
    __shared__ int best[4], worst[4];
    const uint32_t wave = uniform(threadIdx.x >> 6), lane = lane_id();
    const bool of_w = blockIdx.x >= RANGE_BLOCKS;
    const uint32_t block = of_w ? blockIdx.x - RANGE_BLOCKS : blockIdx.x, count = of_w ? targets.vocab : rows;
    const T *const m = of_w ? w : x;
    const uint64_t stride = of_w ? w_stride : x_stride;
    int most = NO_RANGE, least = -NO_RANGE;
    if (of_w ? to.w != nullptr || to.entry != nullptr : to.x != nullptr) {
        for (uint32_t row = block * 4 + wave; row < count; row += RANGE_BLOCKS * 4) {
            uint32_t top = 0;
            for (uint32_t c = lane * 8; c < cols; c += 512) {
                float v[8];
                unpack8(load8(m + row * stride + c, live8(c, cols)), v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t u = __float_as_uint(v[i]) & 0x7FFFFFFFu;
                    top = u < 0x7F800000u ? max(top, u) : top;
                }
            }
            int e = wave_max(exponent_of(top));
            if (!of_w) {
                int power = 0;
                if (row_info) {
                    HeadRow h;
                    const float up = target_of(targets, row) < targets.vocab ? dloss ? dloss[row] : 1.0f : 0.0f;
                    const float all = up + (dlse ? dlse[row] : 0.0f);
                    const float larger = max(__builtin_fabsf(up), __builtin_fabsf(all));
                    const bool plain = larger > 0.0f && larger < __builtin_inff();
                    power = plain ? exponent_of(__float_as_uint(larger)) : 0;
                    h.lse = lse[row];
                    h.pull = times_power(all, GRAD_TOP - power);
                    h.push = times_power(up, GRAD_TOP - power);
                    h.power = power;
                    if (lane == 0) row_info[row] = h;
                    // (a row that nothing arrives at asks for no range)
                    if (up == 0.0f && all == 0.0f) power = NO_RANGE;
                }
                if (lane == 0) to.row[row] = e;
                e = e <= NO_RANGE / 2 || power <= NO_RANGE / 2 ? NO_RANGE : e + power;
            } else {
                if (to.entry && lane == 0) to.entry[row] = e;
                least = e > NO_RANGE / 2 ? min(least, e) : least;
            }
            most = max(most, e);
        }
    }
    if (lane == 0) {
        best[wave] = most;
        worst[wave] = least;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        const int v = max(max(best[0], best[1]), max(best[2], best[3]));
        if (of_w && to.w) to.w[block] = v;
        if (of_w && to.w_least) to.w_least[block] = min(min(worst[0], worst[1]), min(worst[2], worst[3]));
        if (!of_w && to.x) to.x[block] = v;
    }
}

enum CopyKind {
    COPY_PLAIN,      // 16-bit values as they are, in rows whose length is a multiple of eight
    COPY_ROWS,       // halves of a matrix, each row scaled by itself (and once more, all by the same power; of an even one this alone)
    COPY_WEIGHED,    // ... all by the same power, and each row times its own
    COPY_ALL,        // ... all by the same power
};

struct CopyJob {
    const void *from;
    uint64_t stride;
    uint16_t *hi, *lo;      // lo: absent where one part is wanted
    uint16_t *all_hi, *all_lo;      // COPY_ROWS: of the other copy, or absent
    const int *powers;      // COPY_ROWS: of the rows
    uint32_t rows, blocks;
    int32_t kind;
};
constexpr int COPY_JOBS = 4;
struct CopyJobs {
    CopyJob job[COPY_JOBS];
    uint32_t count, cols, pieces;      // of every matrix: columns, and eights of them
};

// Operands in the form that the products read.  Eight columns a lane; columns up to the next multiple of eight are zeros.  Bound by memory:
// a bfloat16 W of 32768 x 4096 and x of 8192 x 4096 into halves, 671 MB, 107 us (6.3 TB/s, part of it from cache).
template <class T>
__global__ __launch_bounds__(256) void k_head_copy(CopyJobs jobs, Ranges ranges, const HeadRow *row_info, Scales *scales)
{
    __shared__ int best[4], worst[4];
    uint32_t block = blockIdx.x, which = 0;
    CopyJob j = jobs.job[0];
#pragma unroll
    for (int i = 1; i < COPY_JOBS; ++i)
        if (which + 1 < jobs.count && block >= j.blocks) {
            block -= j.blocks;
            j = jobs.job[i];
            which = i;
        }
    int all = 0;
    bool even = false;
    if (j.kind == COPY_WEIGHED || j.kind == COPY_ALL || j.all_hi) {
        const int *const r = j.kind == COPY_WEIGHED ? ranges.x : ranges.w;
        int most = NO_RANGE, least = -NO_RANGE;
#pragma unroll
        for (uint32_t k = 0; k < RANGE_BLOCKS; k += 256) {
            most = max(most, r[k + threadIdx.x]);
            if (j.all_hi) least = min(least, ranges.w_least[k + threadIdx.x]);
        }
        most = wave_max(most);
        least = -wave_max(-least);
        if (lane_id() == 0) {
            best[threadIdx.x >> 6] = most;
            worst[threadIdx.x >> 6] = least;
        }
        __syncthreads();
        most = max(max(best[0], best[1]), max(best[2], best[3]));
        least = min(min(worst[0], worst[1]), min(worst[2], worst[3]));
        all = scale_of(most);
        if (j.all_hi) {
            even = most - least <= SPREAD;
            if (block == 0 && threadIdx.x == 0) scales->even = even;
        }
        if (block == 0 && threadIdx.x == 0) (j.kind == COPY_WEIGHED ? scales->x : scales->w) = all;
    }
    const uint64_t step = (uint64_t)j.blocks * 256, end = (uint64_t)j.rows * jobs.pieces;
    for (uint64_t at = (uint64_t)block * 256 + threadIdx.x; at < end; at += step) {
        const uint32_t row = (uint32_t)(at / jobs.pieces), c = (uint32_t)(at - (uint64_t)row * jobs.pieces) * 8;
        const Raw8<T> raw = load8((const T *)j.from + row * j.stride + c, live8(c, jobs.cols));
        u32x4 h, l;
        if (j.kind == COPY_PLAIN) {
            __builtin_memcpy(&h, &raw, 16);
            *(u32x4 *)(j.hi + at * 8) = h;
            continue;
        }
        int e = all;
        float v[8];
        unpack8(raw, v);
        if (j.kind == COPY_ROWS && !even) {
            if (j.all_hi) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = times_power(v[i], all);
                halves8<LOW>(w, h, l);
                *(u32x4 *)(j.all_hi + at * 8) = h;
                *(u32x4 *)(j.all_lo + at * 8) = l;
            }
            e = scale_of(j.powers[row]);
        }
        if (j.kind == COPY_WEIGHED) {
            const HeadRow r = row_info[row];
            e = all + r.power;
            if (nothing_arrives(r)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = times_power(v[i], e);
        halves8<LOW>(v, h, l);
        *(u32x4 *)(j.hi + at * 8) = h;
        if (j.lo) *(u32x4 *)(j.lo + at * 8) = l;
    }
}

// ---------------------------------------------------------------------------
// logits
// ---------------------------------------------------------------------------

struct LogitArgs {
    Side w, x;
    uint32_t cols, kind;             // of the products
    uint32_t rows, vocab, first, end;      // entries of this launch
    uint32_t v_tiles, t_tiles;
    const float *bias;
    Targets targets;
    const int *x_powers, *w_powers;  // exponents of x's and W's rows, fp32 only
    const Scales *scales;            // where dx takes a copy of its own of such a W
    // forward: a row's maximum and sum, for each tile of the vocabulary; the target's logit
    float2 *stats;
    float *target_logit;
    // backward
    const HeadRow *row_info;
    uint16_t *grad[2];               // rows x grad_stride each
    uint64_t grad_stride;
    float *bias_parts;               // t_tiles x grad_stride
};

// Two parts of a row's sum of exponentials, each a maximum and the sum relative to it.
__device__ __forceinline__ float2 joined(float2 a, float2 b)
{
    const float most = max(a.x, b.x), from = most == -__builtin_inff() ? 0.0f : most;
    return make_float2(most, a.y * power_of_e(a.x - from) + b.y * power_of_e(b.x - from));
}

// ---------------------------------------------------------------------------
// few rows
// ---------------------------------------------------------------------------
// Up to 32 rows are one square's columns, and every call is a pass or two over W: what counts is to read it once, as it is.  A
// workgroup takes 32 entries, its fragments straight from memory (any alignment, any type; fp32 in three bfloat16 parts, whose six
// largest products leave 2^-23 of a product out): a copy of W in another form would move it twice more.  Its wavefronts take the
// columns in turn, so that enough loads are in flight where W has few rows.

constexpr uint32_t FEW_ROWS = 32, FEW_WAVES = 4;

// Eight values in three parts, each taken off the rest by truncation: exact but for the smallest numbers.
__device__ __forceinline__ void three_parts(const float (&v)[8], u32x4 (&part)[3])
{
    float left[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) left[i] = v[i];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            part[p][i] = (__float_as_uint(left[2 * i]) >> 16) | (__float_as_uint(left[2 * i + 1]) & 0xFFFF0000u);
#pragma unroll
        for (int i = 0; i < 8; ++i) left[i] -= __uint_as_float(__float_as_uint(left[i]) & 0xFFFF0000u);
    }
}

template <class T> __device__ __forceinline__ void multiply8(const Raw8<T> &a, const Raw8<T> &b, f32x16 &sums)
{
    if constexpr (sizeof(T) == 4) {
        float v[8];
        u32x4 x[3], y[3];
        unpack8(a, v);
        three_parts(v, x);
        unpack8(b, v);
        three_parts(v, y);
#pragma unroll
        for (int all = 2; all >= 0; --all)
#pragma unroll
            for (int i = 0; i <= all; ++i) sums = matrix_unit_of<bf16>(x[i], y[all - i], sums);
    } else {
        u32x4 x, y;
        __builtin_memcpy(&x, &a, 16);
        __builtin_memcpy(&y, &b, 16);
        sums = matrix_unit_of<T>(x, y, sums);
    }
}

// 32 rows of w by 32 of x, over all columns; the first wavefront gets the sums.  (Rows beyond the last are the last.)
template <class T>
__device__ __forceinline__ void few_sums(const Side &w, uint32_t w_first, const Side &x, uint32_t cols, float (&part)[FEW_WAVES - 1][16][64],
                                         f32x16 &sums)
{
    constexpr uint32_t EACH = sizeof(T) == 4 ? 4 : 8, CHUNK = 16 * EACH, TURN = FEW_WAVES * CHUNK;
    const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6), behind = 8 * (lane >> 5);
    const T *const pw = (const T *)w.part[0] + min(w_first + (lane & 31u), w.size - 1u) * w.stride;
    const T *const px = (const T *)x.part[0] + min(lane & 31u, x.size - 1u) * x.stride;
#pragma unroll
    for (int r = 0; r < 16; ++r) sums[r] = 0.0f;
    Raw8<T> a[2][EACH], b[2][EACH];
    auto fetch = [&](int to, uint32_t k) {
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) {
            a[to][i] = load8(pw + k + 16 * i + behind, 8);
            b[to][i] = load8(px + k + 16 * i + behind, 8);
        }
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (uint32_t i = 0; i < EACH; ++i) multiply8<T>(a[from][i], b[from][i], sums);
    };
    const uint32_t whole = cols / CHUNK * CHUNK, first = wave * CHUNK;
    if (first < whole) fetch(0, first);
    for (uint32_t k = first; k < whole; k += 2 * TURN) {
        if (k + TURN < whole) fetch(1, k + TURN);
        multiply(0);
        if (k + TURN < whole) {
            if (k + 2 * TURN < whole) fetch(0, k + 2 * TURN);
            multiply(1);
        }
    }
    for (uint32_t k = whole + 16 * wave; k < cols; k += 16 * FEW_WAVES) {
        const uint32_t c = k + behind, n = live8(c, cols);
        multiply8<T>(load8(pw + (n ? c : 0u), n), load8(px + (n ? c : 0u), n), sums);
    }
    if (wave) {
#pragma unroll
        for (int r = 0; r < 16; ++r) part[wave - 1][r][lane] = sums[r];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (uint32_t i = 0; i < FEW_WAVES - 1; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sums[r] += part[i][r][lane];
    }
}

// dx of few rows, a part of it: sums over `chunk` entries, in fp32, of the logits' gradient (both halves) and W as it is.  256 columns to a
// workgroup, four a lane, its wavefronts taking 32 entries in turn, of which the gradient is in LDS.
constexpr uint32_t FEW_BLOCK = 32;
template <class T> __device__ __forceinline__ void load4(const T *p, uint32_t n, float (&v)[4])
{
    if (n >= 4) {
        T t[4];
        if constexpr (sizeof(T) == 4) {
            const f32x4_any q = *(const f32x4_any *)p;
            __builtin_memcpy(t, &q, 16);
        } else {
            const u32x2_any q = *(const u32x2_any *)p;
            __builtin_memcpy(t, &q, 8);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_float(t[i]);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[i] = i < n ? to_float(p[i]) : 0.0f;
    }
}
template <class T, uint32_t ROWS>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_head_few_dx(const T *w, uint64_t w_stride, uint32_t count, uint32_t cols, const uint16_t *hi,
                                                                const uint16_t *lo, uint64_t grad_stride, uint32_t rows, uint32_t chunk,
                                                                float *sums, uint32_t add)
{
    constexpr uint32_t AHEAD = 8;
    __shared__ union {
        __attribute__((aligned(16))) float grad[FEW_WAVES][FEW_BLOCK][ROWS];
        float part[FEW_WAVES / 2][ROWS * 4][64];
    } lds;
    const uint32_t lane = lane_id(), wave = uniform(threadIdx.x >> 6), c = blockIdx.x * 256 + lane * 4, n = c < cols ? min(4u, cols - c) : 0u;
    const uint32_t first = blockIdx.y * chunk, end = min(first + chunk, count);
    float (*const grad)[ROWS] = lds.grad[wave];
    float s[ROWS][4];
#pragma unroll
    for (uint32_t t = 0; t < ROWS; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.0f;
    for (uint32_t turn = first; turn < end; turn += FEW_WAVES * FEW_BLOCK) {
        const uint32_t v0 = turn + wave * FEW_BLOCK;
        __syncthreads();
#pragma unroll
        for (uint32_t t = 0; t < ROWS; t += 2) {
            const uint32_t row = t + (lane >> 5), v = v0 + (lane & 31u);
            const bool in = row < rows && v < end;
            const uint64_t at = in ? row * grad_stride + v : 0u;
            grad[lane & 31u][row] = in ? half_value(hi[at]) + half_value(lo[at]) * (1.0f / (1u << LOW)) : 0.0f;
        }
        __syncthreads();
        for (uint32_t v = 0; v < FEW_BLOCK && v0 + v < end; v += AHEAD) {
            float x[AHEAD][4];
#pragma unroll
            for (uint32_t i = 0; i < AHEAD; ++i) {
                const bool in = v0 + v + i < end;      // (beyond the end the gradient is 0, and W is not read)
                load4(w + (n && in ? (v0 + v + i) * w_stride + c : 0u), in ? n : 0u, x[i]);
            }
#pragma unroll
            for (uint32_t i = 0; i < AHEAD; ++i)
#pragma unroll
                for (uint32_t t = 0; t < ROWS; t += 4) {
                    const f32x4 g = *(const f32x4 *)&grad[v + i][t];
                    const float q[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
                        for (uint32_t e = 0; e < 4; ++e) s[t + k][e] = __builtin_fmaf(q[k], x[i][e], s[t + k][e]);
                }
        }
    }
    // the wavefronts' sums, by halves
#pragma unroll
    for (uint32_t by = FEW_WAVES / 2; by; by >>= 1) {
        __syncthreads();
        if (wave >= by && wave < 2 * by) {
#pragma unroll
            for (uint32_t t = 0; t < ROWS; ++t)
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) lds.part[wave - by][4 * t + e][lane] = s[t][e];
        }
        __syncthreads();
        if (wave < by) {
#pragma unroll
            for (uint32_t t = 0; t < ROWS; ++t)
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) s[t][e] += lds.part[wave][4 * t + e][lane];
        }
    }
    if (wave) return;
#pragma unroll
    for (uint32_t t = 0; t < ROWS; ++t) {
        if (t >= rows) continue;
        float *const to = sums + ((uint64_t)blockIdx.y * rows + t) * cols + c;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e)
            if (e < n) to[e] = add ? to[e] + s[t][e] : s[t][e];
    }
}

// Entries (m) and rows (n) of a tile.  E: the operands' type as they are staged; STAGES = 0: as they are read, a square to a wavefront.
// Bound by the matrix units: of 8192 x 4096 x 32768 (2.2 TFLOP, bfloat16) 1718 us, 1280 TFLOP/s, with the gradient's halves written
// (1.1 GB) 1853; of 8192 x 768 x 30522 388 and 547, since 12 steps a tile hide less of its epilogue.  One row of 768 columns: by W's reading,
// 47 MB in 10.7 us.  No branch in the epilogue but for tiles at the edge or with a target: with them 16384 x 768 x 30522 760 us, without 671.
template <class E, uint32_t M, uint32_t N, uint32_t WAVES_M, uint32_t WAVES_N, uint32_t STAGES, bool BACK>
__global__ __launch_bounds__(STAGES ? WAVES_M *WAVES_N * 64 : FEW_WAVES * 64, 2) void k_head_logits(LogitArgs a)
{
    typedef Product<E, M, N, WAVES_M, WAVES_N, false, false, STAGES, PRODUCT_STEP, __is_same(E, f16) ? LOW : 0> P;
    __shared__ __attribute__((aligned(16))) typename P::Lds lds;
    const TilePlace place = place_of_tile(tile_of_block(blockIdx.x, gridDim.x), a.v_tiles, a.t_tiles);
    const uint32_t tile_v = place.m, tile_t = place.n;
    const uint32_t v0 = a.first + tile_v * M, t0 = tile_t * N;
    __shared__ __attribute__((aligned(16))) float bias[M];
    if (a.bias) {      // (read behind the product's barriers)
        for (uint32_t m = threadIdx.x; m < M; m += P::THREADS) bias[m] = a.bias[min(v0 + m, a.end - 1u)];
    }
    constexpr bool SPLIT = STAGES > 0 && __is_same(E, f16);      // (fp32 operands may have come in halves)
    __shared__ __attribute__((aligned(16))) int w_power[SPLIT ? M : 4];
    if constexpr (SPLIT) {
        if (a.w_powers) {
            const bool even = a.scales && a.scales->even;
            for (uint32_t m = threadIdx.x; m < M; m += P::THREADS)
                w_power[m] = even ? -a.scales->w : -scale_of(a.w_powers[min(v0 + m, a.end - 1u)]);
        }
    }
    typename P::Sums z;
    if constexpr (STAGES == 0) {
        __shared__ float part[FEW_WAVES - 1][16][64];
        few_sums<E>(a.w, v0, a.x, a.cols, part, z[0][0]);
        if (threadIdx.x >= 64) return;      // (the rest is a wavefront's work)
    } else {
        P::run(lds, a.w, a.x, v0, t0, 0, a.cols, a.kind, z);
    }

    const uint32_t lane = lane_id(), half = lane >> 5, wave = uniform(threadIdx.x >> 6);
    // this lane's first entry of the tile; the others are row_in_square(r) + 32 i behind it, `left` of them are there
    const uint32_t v_lane = v0 + P::wave_m() + 4 * half, left = a.end - min(v_lane, a.end);
    const bool edge = v0 + M > a.end;
    uint32_t target[P::J];
    bool here[P::J];
#pragma unroll
    for (uint32_t j = 0; j < P::J; ++j) {
        const uint32_t t = t0 + P::wave_n() + 32 * j + (lane & 31u);
        here[j] = t < a.rows;
        target[j] = here[j] ? target_of(a.targets, t) : a.vocab;
        if constexpr (SPLIT) {
            if (a.x_powers) {
                const int e = here[j] ? -scale_of(a.x_powers[t]) : 0;
#pragma unroll
                for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
                    for (uint32_t r = 0; r < 16; ++r)
                        z[i][j][r] = times_power(z[i][j][r], e + w_power[P::wave_m() + 32 * i + row_in_square(r) + 4 * half]);
            }
        }
    }
    if (a.bias) {
#pragma unroll
        for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
            for (uint32_t g = 0; g < 4; ++g) {
                const f32x4 b = *(const f32x4 *)(bias + P::wave_m() + 32 * i + 8 * g + 4 * half);
#pragma unroll
                for (uint32_t j = 0; j < P::J; ++j) {
                    z[i][j][4 * g] += b.x;
                    z[i][j][4 * g + 1] += b.y;
                    z[i][j][4 * g + 2] += b.z;
                    z[i][j][4 * g + 3] += b.w;
                }
            }
    }
    if constexpr (!BACK) {
        P::sync();      // nobody reads operands any more
        float2(*const part)[N] = (float2(*)[N])&lds;
        if (edge) {
#pragma unroll
            for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
                for (uint32_t j = 0; j < P::J; ++j)
#pragma unroll
                    for (uint32_t r = 0; r < 16; ++r) z[i][j][r] = 32 * i + row_in_square(r) < left ? z[i][j][r] : -__builtin_inff();
        }
#pragma unroll
        for (uint32_t j = 0; j < P::J; ++j) {
            const uint32_t n = P::wave_n() + 32 * j + (lane & 31u), t = t0 + n;
            const uint32_t aim = target[j] - v_lane;      // (where the target lies, if it lies here)
            if (ballot64(aim < 32 * P::I)) {
                float hit = 0.0f;
                bool found = false;
#pragma unroll
                for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
                    for (uint32_t r = 0; r < 16; ++r) {
                        const bool is = 32 * i + row_in_square(r) == aim;
                        hit = is ? z[i][j][r] : hit;
                        found |= is;
                    }
                if (found && here[j]) a.target_logit[t] = hit;
            }
            float most = -__builtin_inff(), sum = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) most = max(most, z[i][j][r]);
            most = max(most, other_half(most));
            const float from = most == -__builtin_inff() ? 0.0f : most;
#pragma unroll
            for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) sum += power_of_e(z[i][j][r] - from);
            sum += other_half(sum);
            if (half == 0) part[wave / WAVES_N][n] = make_float2(most, sum);
        }
        P::sync();
        for (uint32_t n = threadIdx.x; n < N; n += P::THREADS) {
            if (t0 + n >= a.rows) continue;
            float2 all = part[0][n];
#pragma unroll
            for (uint32_t w = 1; w < WAVES_M; ++w) all = joined(all, part[w][n]);
            a.stats[(uint64_t)tile_v * a.rows + t0 + n] = all;
        }
    } else {
        float weight[P::J];      // what the bias gradient takes of a row
#pragma unroll
        for (uint32_t j = 0; j < P::J; ++j) {
            const uint32_t t = t0 + P::wave_n() + 32 * j + (lane & 31u);
            HeadRow h = {0.0f, 0.0f, 0.0f, 0};
            if (here[j]) h = a.row_info[t];
            weight[j] = times_power(1.0f, h.power - GRAD_TOP);
            // what is not there counts as a logit of -infinity; so does all of a row that nothing arrives at, whatever its logits are
            const bool none = nothing_arrives(h);
            const uint32_t there = none ? 0u : left;
            if (none) h.lse = 0.0f;
            const uint32_t aim = target[j] - v_lane;
            if (edge || ballot64(none)) {
#pragma unroll
                for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
                    for (uint32_t r = 0; r < 16; ++r) z[i][j][r] = 32 * i + row_in_square(r) < there ? z[i][j][r] : -__builtin_inff();
            }
#pragma unroll
            for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
                for (uint32_t r = 0; r < 16; ++r) z[i][j][r] = h.pull * power_of_e(z[i][j][r] - h.lse);
            if (ballot64(aim < 32 * P::I)) {
#pragma unroll
                for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
                    for (uint32_t r = 0; r < 16; ++r) z[i][j][r] -= 32 * i + row_in_square(r) == aim ? h.push : 0.0f;
            }
        }
        P::by_columns(lds, z, [&](uint32_t m, uint32_t n, const float (&v)[8]) {
            const uint32_t t = t0 + n, at_v = v0 - a.first + m;
            if (t >= a.rows || at_v >= a.grad_stride) return;
            u32x4 hi, lo;
            halves8<LOW>(v, hi, lo);
            *(u32x4 *)(a.grad[0] + t * a.grad_stride + at_v) = hi;
            *(u32x4 *)(a.grad[1] + t * a.grad_stride + at_v) = lo;
        });
        if (a.bias_parts) {
            P::sync();
            float(*const part)[M] = (float(*)[M])&lds;
            float column[P::I * 16];      // the bias gradient's sums over this lane's rows
#pragma unroll
            for (uint32_t k = 0; k < P::I * 16; ++k) {
                column[k] = z[k / 16][0][k % 16] * weight[0];
#pragma unroll
                for (uint32_t j = 1; j < P::J; ++j) column[k] = __builtin_fmaf(z[k / 16][j][k % 16], weight[j], column[k]);
            }
            // over 32 lanes: of every pair of lanes each takes half of the entries, until one or two are left
            uint32_t entry = 0;
#pragma unroll
            for (uint32_t by = 1, left = P::I * 16; by < 32; by <<= 1) {
                const bool upper = (lane & by) != 0;
                const uint32_t keep = left > 1 ? left / 2 : 1;
#pragma unroll
                for (uint32_t k = 0; k < P::I * 8; ++k) {
                    if (k >= keep) continue;
                    const float mine = left > 1 && upper ? column[k + keep] : column[k], theirs = left > 1 && !upper ? column[k + keep] : column[k];
                    column[k] = mine + __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute((int)((lane ^ by) << 2), (int)__float_as_uint(theirs)));
                }
                entry += left > 1 && upper ? keep : 0u;
                left = keep;
            }
#pragma unroll
            for (uint32_t k = 0; k < (P::I > 2 ? P::I / 2 : 1); ++k)
                part[wave % WAVES_N][P::wave_m() + 32 * ((entry + k) >> 4) + row_in_square((entry + k) & 15u) + 4 * half] = column[k];
            P::sync();
            for (uint32_t m = threadIdx.x; m < M; m += P::THREADS) {
                const uint32_t v = v0 - a.first + m;
                if (v >= a.grad_stride) continue;
                float s = part[0][m];
#pragma unroll
                for (uint32_t w = 1; w < WAVES_N; ++w) s += part[w][m];
                a.bias_parts[tile_t * a.grad_stride + v] = s;
            }
        }
    }
}

// A row's lse and loss from its tiles' parts (8 bytes each: 3 to 7 us, most of it the launch).
// `apart` lanes a row (a power of two), 256 / apart rows.
__global__ __launch_bounds__(256) void k_head_loss(const float2 *stats, const float *target_logit, Targets targets, uint32_t rows,
                                                   uint32_t tiles, uint32_t apart, float *loss, float *lse)
{
    __shared__ float2 part[256];
    const uint32_t per = 256 / apart, n = threadIdx.x % per, group = threadIdx.x / per;
    const uint32_t t = blockIdx.x * per + n, row = min(t, rows - 1u);
    float2 all = make_float2(-__builtin_inff(), 0.0f);
    for (uint32_t i = group; i < tiles; i += 4 * apart) {
        float2 s[4];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) s[k] = stats[(uint64_t)min(i + k * apart, tiles - 1u) * rows + row];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
            if (i + k * apart < tiles) all = joined(all, s[k]);
    }
    part[threadIdx.x] = all;
    for (uint32_t by = apart / 2; by; by >>= 1) {
        __syncthreads();
        if (group < by) part[threadIdx.x] = joined(part[threadIdx.x], part[threadIdx.x + by * per]);
    }
    if (group || t >= rows) return;
    all = part[threadIdx.x];
    const float l = all.x == -__builtin_inff() && all.y == 0.0f ? all.x : all.x + logf(all.y);
    lse[t] = l;
    if (loss) loss[t] = target_of(targets, t) < targets.vocab ? l - target_logit[t] : 0.0f;
}

// ---------------------------------------------------------------------------
// gradients
// ---------------------------------------------------------------------------

struct GradientArgs {
    Side a, b;
    uint32_t depth, split_depth, kind;      // the sum's length, and of a split of it
    uint32_t m_tiles, n_tiles, splits;
    uint32_t m, n;
    float *out;              // whole: the result; otherwise splits x m x n of partial sums
    uint64_t out_stride;
    uint32_t add, whole;
    const Scales *scales;    // whole: x's exponent comes off
    const uint16_t *even[2]; // of b, what takes its parts' place where W is even; or absent
};

// A tile of dx (of a piece's entries) or dweight (TURN_A: the first operand's k lies outside; the second's always does).  Bound by the matrix units:
// of 8192 x 4096 x 32768, dx 1753 us (1254 TFLOP/s), dweight, of two halves, 3622 (1214).  Of 8192 x 768 x 30522 dx 379 and dweight 742:
// 256 x 128, two workgroups to a compute unit, so that one's epilogue overlaps the other's product; 256 x 256 takes 882.
template <uint32_t M, uint32_t N, uint32_t WAVES_M, uint32_t WAVES_N, uint32_t STAGES, bool TURN_A> struct GradientTile {
    typedef Product<f16, M, N, WAVES_M, WAVES_N, TURN_A, true, STAGES, M == 256 && N == 128 ? 32 : PRODUCT_STEP, LOW> P;
    static __device__ __forceinline__ void run(typename P::Lds &lds, const GradientArgs &a, uint32_t at);
};
template <uint32_t M, uint32_t N, uint32_t WAVES_M, uint32_t WAVES_N, uint32_t STAGES, bool TURN_A>
__device__ __forceinline__ void GradientTile<M, N, WAVES_M, WAVES_N, STAGES, TURN_A>::run(typename P::Lds &lds, const GradientArgs &a, uint32_t at)
{
    const uint32_t tiles = a.m_tiles * a.n_tiles;
    const uint32_t split = at / tiles;
    const TilePlace place = place_of_tile(at - split * tiles, a.m_tiles, a.n_tiles);
    const uint32_t tile_m = place.m, tile_n = place.n;
    const uint32_t first = min(split * a.split_depth, a.depth), end = min(first + a.split_depth, a.depth);
    float *const out = a.out + (a.whole ? 0u : (uint64_t)split * a.m * a.out_stride);
    typename P::Sums s;
    Side b = a.b;
    if constexpr (!TURN_A) {
        if (a.even[0] && a.scales->even) {
            b.part[0] = a.even[0];
            b.part[1] = a.even[1];
        }
    }
    P::run(lds, a.a, b, tile_m * M, tile_n * N, first, end, a.kind, s);
    const int e = a.whole ? -GRAD_TOP - a.scales->x : 0;
    f32x4 old[2 * P::PASSES];
    P::by_fours(lds, s, [&](uint32_t p, uint32_t row, uint32_t col) {
        const uint32_t m = tile_m * M + row, n = tile_n * N + col;
        if (a.add && m < a.m && n + 4 <= a.n) old[p] = *(const f32x4_any *)(out + m * a.out_stride + n);
    }, [&](uint32_t p, uint32_t row, uint32_t col, const f32x4 &v) {
        const uint32_t m = tile_m * M + row, n = tile_n * N + col;
        if (m >= a.m || n >= a.n) return;
        float *const to = out + m * a.out_stride + n;
        f32x4_any w;
        w.x = times_power(v.x, e); w.y = times_power(v.y, e); w.z = times_power(v.z, e); w.w = times_power(v.w, e);
        if (n + 4 <= a.n) {
            if (a.add) w += old[p];
            __builtin_nontemporal_store(w, (f32x4_any *)to);
        } else {
            to[0] = a.add ? to[0] + w.x : w.x;
            if (n + 1 < a.n) to[1] = a.add ? to[1] + w.y : w.y;
            if (n + 2 < a.n) to[2] = a.add ? to[2] + w.z : w.z;
        }
    });
}

template <uint32_t M, uint32_t N, uint32_t WAVES_M, uint32_t WAVES_N, uint32_t STAGES, bool TURN_A>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64, 2) void k_head_product(GradientArgs a)
{
    typedef GradientTile<M, N, WAVES_M, WAVES_N, STAGES, TURN_A> G;
    __shared__ __attribute__((aligned(16))) typename G::P::Lds lds;
    G::run(lds, a, tile_of_block(blockIdx.x, gridDim.x));
}

struct BiasArgs {
    const float *parts;      // tiles x stride
    uint32_t tiles, count, add;
    uint64_t stride;
    float *out;
};
// dbias: the tiles' sums, 64 entries to a workgroup, four lanes each.
__device__ __forceinline__ void sum_bias(const BiasArgs &a, uint32_t block, float *sums)
{
    const uint32_t v = block * 64 + (threadIdx.x & 63u), at = min(v, a.count - 1u);
    float s = 0.0f;
    for (uint32_t i = threadIdx.x >> 6; i < a.tiles; i += 32) {
        float w[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) w[k] = a.parts[min(i + 4 * k, a.tiles - 1u) * a.stride + at];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) s += i + 4 * k < a.tiles ? w[k] : 0.0f;
    }
    sums[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x >= 64 || v >= a.count) return;
    s = (s + sums[threadIdx.x + 64]) + (sums[threadIdx.x + 128] + sums[threadIdx.x + 192]);
    a.out[v] = a.add ? a.out[v] + s : s;
}
__global__ __launch_bounds__(256) void k_head_dbias(BiasArgs a)
{
    __shared__ float sums[256];
    sum_bias(a, blockIdx.x, sums);
}

// Gradients of little work in one launch: tiles of dweight, tiles of dx, and the bias gradient's sums.  Bound by the latency of few steps, so
// that one beside the other costs little: 300 x 333 x 1009 of fp32 10 us, in three launches 8.4, 8.3 and 1.3 and what lies between them.
__global__ __launch_bounds__(256, 2) void k_head_gradients(GradientArgs dw, GradientArgs dx, BiasArgs bias, uint32_t dw_blocks, uint32_t dx_blocks)
{
    typedef GradientTile<64, 64, 2, 2, 4, true> W;
    typedef GradientTile<64, 64, 2, 2, 4, false> X;
    __shared__ __attribute__((aligned(16))) union {
        typename W::P::Lds w;
        typename X::P::Lds x;
        float sums[256];
    } lds;
    const uint32_t block = blockIdx.x;
    if (block < dw_blocks) W::run(lds.w, dw, tile_of_block(block, dw_blocks));
    else if (block < dw_blocks + dx_blocks) X::run(lds.x, dx, tile_of_block(block - dw_blocks, dx_blocks));
    else sum_bias(bias, block - dw_blocks - dx_blocks, lds.sums);
}

// dx: the splits' sums, times the row's power, W's taken off.  Eight columns a lane; GROUPS lanes take the splits in turn.  Bound by
// memory: 8192 x 4096 of one sum into bfloat16, 201 MB, 36 us (5.6 TB/s).
template <class T, uint32_t GROUPS>
__global__ __launch_bounds__(256) void k_head_dx(const float *sums, uint32_t splits, uint32_t rows, uint32_t cols, const HeadRow *row_info,
                                                 const Scales *scales, T *dx, uint64_t dx_stride)
{
    constexpr uint32_t PER = 256 / GROUPS;
    __shared__ float part[GROUPS][8][PER];
    const uint32_t place = threadIdx.x % PER, group = threadIdx.x / PER;
    const uint64_t at = (uint64_t)blockIdx.x * PER + place, pieces = (cols + 7) / 8;
    const uint64_t row = at / pieces;
    const uint32_t c = (uint32_t)(at - row * pieces) * 8, n = row < rows ? live8(c, cols) : 0u;
    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    const uint64_t apart = (uint64_t)rows * cols;
    const float *const p = sums + (n ? row * cols + c : 0u);
    for (uint32_t s = group; s < splits; s += 4 * GROUPS) {
        float w[4][8];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) load8_f32(p + min(s + k * GROUPS, splits - 1u) * apart, n, w[k]);
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += s + k * GROUPS < splits ? w[k][i] : 0.0f;
    }
    if constexpr (GROUPS > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) part[group][i][place] = v[i];
        __syncthreads();
        if (group) return;
#pragma unroll
        for (uint32_t g = 1; g < GROUPS; ++g)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += part[g][i][place];
    }
    if (n == 0) return;
    const int e = row_info[row].power - GRAD_TOP - (scales ? scales->w : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = times_power(v[i], e);
    store8(dx + row * dx_stride, c, n, v);
}

// dweight: the splits' sums, x's exponent taken off (no splits: zeros).
constexpr uint32_t DWEIGHT_BLOCKS = 1u << 16;      // at most
__global__ __launch_bounds__(256) void k_head_dweight(const float *sums, uint32_t splits, uint32_t rows, uint32_t cols,
                                                      const Scales *scales, float *out, uint64_t out_stride, uint32_t add)
{
    const uint64_t end = (uint64_t)rows * cols;
    for (uint64_t at = blockIdx.x * 256 + threadIdx.x; at < end; at += gridDim.x * 256) {
        const uint64_t row = at / cols;
        float v = 0.0f;
        for (uint32_t s = 0; s < splits; ++s) v += sums[s * end + at];
        if (splits) v = times_power(v, -GRAD_TOP - scales->x);
        float *const p = out + row * out_stride + (at - row * cols);
        *p = add ? *p + v : v;
    }
}
static uint32_t dweight_blocks(uint32_t rows, uint32_t cols)
{
    const uint64_t n = ((uint64_t)rows * cols + 255) / 256;
    return n < DWEIGHT_BLOCKS ? (uint32_t)n : DWEIGHT_BLOCKS;
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

enum { TILE_FEW = PRODUCT_TILES, TILE_DIRECT };      // 128 entries, 32 rows; 32 entries, 32 rows, as they are
struct TileSize { uint32_t m, n; };
static TileSize size_of(int tile) { return tile == TILE_FEW ? TileSize{128, FEW_ROWS} : tile == TILE_DIRECT ? TileSize{32, FEW_ROWS} : TileSize{tile_high(tile), tile_wide(tile)}; }
static uint32_t steps_of(uint32_t depth, uint32_t kind) { return tiles_of(depth, PRODUCT_STEP) * (kind == ONE_PAIR ? 1 : kind == FIRST_IN_TWO ? 2 : 3); }
static int logits_tile(uint32_t vocab, uint32_t rows, uint32_t steps)
{
    float us = 0.0f;
    return product_tile([=](uint32_t high, uint32_t wide) { return (uint64_t)tiles_of(vocab, high) * tiles_of(rows, wide); }, steps, TILE_256, us);
}
// A gradient's product: its tile, and how many splits of the sum are added up by a launch of their own.
struct ProductPlan {
    int tile;
    uint32_t splits, split_depth, kind;
};
static ProductPlan product_plan(uint32_t m, uint32_t n, uint32_t depth, uint32_t kind, int more)
{
    ProductPlan best = {};
    float least = 0.0f;
    const uint32_t steps = depth ? tiles_of(depth, PRODUCT_STEP) : 1u, most = splits_tried(steps, 16);
    for (uint32_t s = 1; s <= most; ++s) {
        const uint32_t each = (steps + s - 1) / s;
        if ((steps + each - 1) / each != s) continue;
        float us = 0.0f;
        const int tile = product_tile([=](uint32_t high, uint32_t wide) { return (uint64_t)tiles_of(m, high) * tiles_of(n, wide) * s; },
                                      steps_of(each * PRODUCT_STEP, kind), more, us);
        if (s > 1) us += 3.0f + (float)s * (float)m * (float)n * 8.0f / 4.5e6f;      // (a split's sums are written and read)
        if (least == 0.0f || us < least || MOST_SPLITS) {
            least = us;
            best = ProductPlan{tile, s, each * PRODUCT_STEP, kind};
        }
    }
    return best;
}

constexpr uint64_t PIECE_BYTES = 1ull << 30;      // of the logits' gradient, at a time

struct HeadPlan {
    bool back, wants_dx, wants_dw;
    bool few, direct, few_dx;        // rows of one square; whose logits, whose dx are taken of W as it is
    bool split, copy_x, copy_w, scale_w;      // which operands are copied, and how
    uint32_t width;                                  // columns, up to a multiple of eight
    uint32_t piece;                                  // entries at a time
    int logits;
    ProductPlan dx, dw;
    uint64_t bytes;
    // sections
    float2 *stats;
    float *target_logit;
    HeadRow *row_info;
    Ranges ranges;
    Scales *scales;
    uint16_t *x[2], *x_weighed[2], *w[2], *w_all[2], *grad[2];      // (w_all: fp32's for dx)
    float *bias_parts, *dx_sums, *dw_sums;
};

// Whether a product's loads take the matrix as it is: in pieces of 16 bytes, and (a tile's 256 rows reached by 31 bits) rows not too far apart.
static bool straight_ok(const dgs_matrix &m, uint32_t rows, uint32_t cols)
{
    return cols % 8 == 0 && aligned_to(m.data, 16) && (rows == 1 || (m.stride % 8 == 0 && m.stride < (1u << 21)));
}
static HeadPlan plan_of(const dgs_head_args &p, bool back)
{
    HeadPlan h = {};
    h.back = back;
    h.wants_dx = back && p.dx.data;
    h.wants_dw = back && p.dweight;
    h.width = (p.cols + 7) & ~7u;
    const bool f32 = p.type == DGS_F32;
    const bool staged = straight_ok(p.x, p.rows, p.cols) && straight_ok(p.weight, p.vocab, p.cols);
    h.few = p.rows <= FEW_ROWS;
    h.direct = h.few && (f32 || !staged);
    // (dx alone, bfloat16 W of 32000 x 4096, by few_dx and by the matrix units from a copy of W: 8 rows 140 and 267 us, 16 rows 206 and 287,
    // 32 rows 360 and 278; of 32000 x 1024 16 rows 67 and 67.  fp32 has its halves beyond 32 rows only: 32000 x 4096, 32 rows forward 156 and
    // dx 395, 33 rows 442 and 598)
    h.few_dx = h.few && (f32 || p.rows <= 16);
    h.split = f32 && !h.few;
    h.scale_w = h.wants_dx && (h.split || (p.type == DGS_BF16 && !h.few_dx));
    h.copy_x = !f32 && !h.few && !straight_ok(p.x, p.rows, p.cols);
    h.copy_w = !f32 && !straight_ok(p.weight, p.vocab, p.cols) && (!h.few || (p.type == DGS_F16 && h.wants_dx && !h.few_dx));
    h.logits = h.direct ? TILE_DIRECT : h.few ? TILE_FEW : logits_tile(p.vocab, p.rows, steps_of(p.cols, f32 ? BOTH_IN_TWO : ONE_PAIR));
    Sections s = {(uintptr_t)p.workspace, 0};
    const uint64_t x_bytes = (uint64_t)p.rows * h.width * 2, w_bytes = (uint64_t)p.vocab * h.width * 2;
    const TileSize tile = size_of(h.logits);
    if (!back) {
        h.stats = (float2 *)s.take((uint64_t)tiles_of(p.vocab, tile.m) * p.rows * sizeof(float2));
        h.target_logit = (float *)s.take((uint64_t)p.rows * 4);
    }
    if (back || h.split) {
        h.ranges.row = (int *)s.take((uint64_t)p.rows * 4);
        h.ranges.x = (int *)s.take(RANGE_BLOCKS * 4);
        h.ranges.w = (int *)s.take(RANGE_BLOCKS * 4);
        if (h.split) {
            h.ranges.entry = (int *)s.take((uint64_t)p.vocab * 4);
            h.ranges.w_least = (int *)s.take(RANGE_BLOCKS * 4);
        }
        h.scales = (Scales *)s.take(sizeof(Scales));
        if (!h.scale_w) h.ranges.w = nullptr;
    }
    if (h.split || h.copy_x) h.x[0] = (uint16_t *)s.take(x_bytes);
    if (h.split) h.x[1] = (uint16_t *)s.take(x_bytes);
    if (h.split || h.copy_w) h.w[0] = (uint16_t *)s.take(w_bytes);
    if (h.split) h.w[1] = (uint16_t *)s.take(w_bytes);
    if (h.split && h.wants_dx)
        for (uint16_t *&w : h.w_all) w = (uint16_t *)s.take(w_bytes);
    if (back) {
        h.row_info = (HeadRow *)s.take((uint64_t)p.rows * sizeof(HeadRow));
        if (h.wants_dw) h.x_weighed[0] = (uint16_t *)s.take(x_bytes);
        if (h.wants_dw && f32) h.x_weighed[1] = (uint16_t *)s.take(x_bytes);
        // the logits' gradient: pieces of the vocabulary, whole tiles of it
        uint64_t most = p.rows ? PIECE_BYTES / (4ull * p.rows) & ~255ull : p.vocab;
        if (most < 256) most = 256;
#ifdef DGS_HEAD_PIECE
        most = DGS_HEAD_PIECE;
#endif
        h.piece = most < p.vocab ? (uint32_t)most : p.vocab;
        const uint64_t stride = ((uint64_t)h.piece + 7) & ~7ull;
        h.grad[0] = (uint16_t *)s.take(p.rows * stride * 2);
        h.grad[1] = (uint16_t *)s.take(p.rows * stride * 2);
        if (p.dbias) h.bias_parts = (float *)s.take(tiles_of(p.rows, tile.n) * stride * 4);
        if (h.few_dx) {
            // a turn of the wavefronts' blocks at least, about 2048 workgroups, at most 128 sums a value
            const uint32_t turn = FEW_WAVES * FEW_BLOCK, across = tiles_of(p.cols, 256);
            const uint32_t most = across > 16 ? (across > 2048 ? 1u : 2048 / across) : 128u;
            const uint32_t each = tiles_of(tiles_of(h.piece, most), turn) * turn;
            h.dx = ProductPlan{0, tiles_of(h.piece, each), each, 0};
        } else h.dx = product_plan(p.rows, p.cols, h.piece, f32 ? BOTH_IN_TWO : p.type == DGS_F16 ? FIRST_IN_TWO : ONE_PAIR, TILE_256);
        h.dw = product_plan(h.piece, p.cols, p.rows, f32 ? BOTH_IN_TWO : FIRST_IN_TWO, TILE_TALL);
        if (h.wants_dx) h.dx_sums = (float *)s.take((uint64_t)h.dx.splits * p.rows * p.cols * 4);
        if (h.wants_dw && h.dw.splits > 1) h.dw_sums = (float *)s.take((uint64_t)h.dw.splits * h.piece * p.cols * 4);
        if (h.scale_w && !f32) h.w[1] = (uint16_t *)s.take(w_bytes);      // (of bfloat16: W in half, for dx)
    }
    h.bytes = s.used ? s.used : 256;
    return h;
}

template <class T> static void prepare(const dgs_head_args &p, const HeadPlan &h, const Targets &targets, hipStream_t st)
{
    if (h.back || h.split)
        hipLaunchKernelGGL(k_head_range<T>, dim3(2 * RANGE_BLOCKS), dim3(256), 0, st, (const T *)p.x.data, p.x.stride,
                           (const T *)p.weight.data, p.weight.stride, p.rows, p.cols, targets, (const float *)p.lse, p.dloss, p.dlse,
                           h.row_info, h.ranges);
    CopyJobs jobs = {};
    jobs.cols = p.cols;
    jobs.pieces = h.width / 8;
    uint32_t blocks = 0;
    auto job = [&](const dgs_matrix &m, uint32_t rows, int kind, uint16_t *hi, uint16_t *lo) {
        const uint64_t n = ((uint64_t)rows * jobs.pieces + 255) / 256;
        const uint32_t b = n < 4096 ? (uint32_t)n : 4096u;
        jobs.job[jobs.count++] = CopyJob{m.data, m.stride, hi, lo, nullptr, nullptr, nullptr, rows, b, kind};
        blocks += b;
    };
    if (h.split) {
        job(p.x, p.rows, COPY_ROWS, h.x[0], h.x[1]);
        jobs.job[0].powers = h.ranges.row;
        job(p.weight, p.vocab, COPY_ROWS, h.w[0], h.w[1]);
        jobs.job[1].powers = h.ranges.entry;
        jobs.job[1].all_hi = h.w_all[0];
        jobs.job[1].all_lo = h.w_all[1];
    } else {
        if (h.copy_x) job(p.x, p.rows, COPY_PLAIN, h.x[0], nullptr);
        if (h.copy_w) job(p.weight, p.vocab, COPY_PLAIN, h.w[0], nullptr);
        if (h.scale_w) job(p.weight, p.vocab, COPY_ALL, h.w[1], nullptr);
    }
    if (h.wants_dw) job(p.x, p.rows, COPY_WEIGHED, h.x_weighed[0], h.x_weighed[1]);
    if (blocks) hipLaunchKernelGGL(k_head_copy<T>, dim3(blocks), dim3(256), 0, st, jobs, h.ranges, (const HeadRow *)h.row_info, h.scales);
}

template <class E, bool BACK> static void logits(const LogitArgs &a, int tile, hipStream_t st)
{
    const dim3 grid(a.v_tiles * a.t_tiles);
    if (tile == TILE_256) hipLaunchKernelGGL((k_head_logits<E, 256, 256, 2, 4, 2, BACK>), grid, dim3(512), 0, st, a);
    else if (tile == TILE_128) hipLaunchKernelGGL((k_head_logits<E, 128, 128, 2, 2, 2, BACK>), grid, dim3(256), 0, st, a);
    else if (tile == TILE_64) hipLaunchKernelGGL((k_head_logits<E, 64, 64, 2, 2, 4, BACK>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_head_logits<E, 128, 32, 4, 1, 3, BACK>), grid, dim3(256), 0, st, a);
}
template <bool BACK> static void logits(const LogitArgs &a, int type, int tile, hipStream_t st)
{
    if (tile == TILE_DIRECT) {
        const dim3 grid(a.v_tiles * a.t_tiles);
        if (type == DGS_F32) hipLaunchKernelGGL((k_head_logits<float, 32, 32, 1, 1, 0, BACK>), grid, dim3(FEW_WAVES * 64), 0, st, a);
        else if (type == DGS_F16) hipLaunchKernelGGL((k_head_logits<f16, 32, 32, 1, 1, 0, BACK>), grid, dim3(FEW_WAVES * 64), 0, st, a);
        else hipLaunchKernelGGL((k_head_logits<bf16, 32, 32, 1, 1, 0, BACK>), grid, dim3(FEW_WAVES * 64), 0, st, a);
        return;
    }
    if (type == DGS_BF16) logits<bf16, BACK>(a, tile, st);
    else logits<f16, BACK>(a, tile, st);
}
template <bool TURN_A> static void product(const GradientArgs &a, int tile, hipStream_t st)
{
    const dim3 grid(a.m_tiles * a.n_tiles * a.splits);
    if (tile == TILE_256) hipLaunchKernelGGL((k_head_product<256, 256, 2, 4, 2, TURN_A>), grid, dim3(512), 0, st, a);
    else if (tile == TILE_TALL) {
        if constexpr (TURN_A) hipLaunchKernelGGL((k_head_product<256, 128, 2, 2, 3, TURN_A>), grid, dim3(256), 0, st, a);
    }
    else if (tile == TILE_128) hipLaunchKernelGGL((k_head_product<128, 128, 2, 2, 2, TURN_A>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_head_product<64, 64, 2, 2, 4, TURN_A>), grid, dim3(256), 0, st, a);
}

template <class T, uint32_t ROWS>
static void few_dx_of(const dgs_head_args &p, const HeadPlan &h, uint32_t first, uint32_t count, uint64_t stride, hipStream_t st)
{
    hipLaunchKernelGGL((k_head_few_dx<T, ROWS>), dim3(tiles_of(p.cols, 256), h.dx.splits), dim3(FEW_WAVES * 64), 0, st,
                       (const T *)p.weight.data + first * p.weight.stride, p.weight.stride, count, p.cols, (const uint16_t *)h.grad[0],
                       (const uint16_t *)h.grad[1], stride, p.rows, h.dx.split_depth, h.dx_sums, (uint32_t)(first != 0));
}
template <class T> static void few_dx_by_rows(const dgs_head_args &p, const HeadPlan &h, uint32_t first, uint32_t count, uint64_t stride, hipStream_t st)
{
    if (p.rows <= 4) few_dx_of<T, 4>(p, h, first, count, stride, st);
    else if (p.rows <= 8) few_dx_of<T, 8>(p, h, first, count, stride, st);
    else if (p.rows <= 16) few_dx_of<T, 16>(p, h, first, count, stride, st);
    else if constexpr (__is_same(T, float)) few_dx_of<T, FEW_ROWS>(p, h, first, count, stride, st);
}
static void few_dx(const dgs_head_args &p, const HeadPlan &h, uint32_t first, uint32_t count, uint64_t stride, hipStream_t st)
{
    if (p.type == DGS_F32) few_dx_by_rows<float>(p, h, first, count, stride, st);
    else if (p.type == DGS_F16) few_dx_by_rows<f16>(p, h, first, count, stride, st);
    else few_dx_by_rows<bf16>(p, h, first, count, stride, st);
}

template <class T> static void finish_dx(const dgs_head_args &p, const HeadPlan &h, const Scales *scales, hipStream_t st)
{
    const uint64_t pieces = (uint64_t)p.rows * ((p.cols + 7) / 8);
    if (h.dx.splits > 16)
        hipLaunchKernelGGL((k_head_dx<T, 8>), dim3((uint32_t)((pieces + 31) / 32)), dim3(256), 0, st, (const float *)h.dx_sums, h.dx.splits,
                           p.rows, p.cols, (const HeadRow *)h.row_info, scales, (T *)p.dx.data, p.dx.stride);
    else
        hipLaunchKernelGGL((k_head_dx<T, 1>), dim3((uint32_t)((pieces + 255) / 256)), dim3(256), 0, st, (const float *)h.dx_sums, h.dx.splits,
                           p.rows, p.cols, (const HeadRow *)h.row_info, scales, (T *)p.dx.data, p.dx.stride);
}

static LogitArgs logit_args(const dgs_head_args &p, const HeadPlan &h, const Targets &targets)
{
    LogitArgs a = {};
    const bool f32 = p.type == DGS_F32;
    const bool own_x = h.split || h.copy_x, own_w = h.split || (h.copy_w && !h.direct);
    a.x = Side{{own_x ? h.x[0] : (const uint16_t *)p.x.data, h.x[1]}, own_x ? h.width : p.x.stride, p.rows};
    a.w = Side{{own_w ? h.w[0] : (const uint16_t *)p.weight.data, h.w[1]}, own_w ? h.width : p.weight.stride, p.vocab};
    a.cols = p.cols;
    a.kind = f32 ? BOTH_IN_TWO : ONE_PAIR;
    a.rows = p.rows;
    a.vocab = p.vocab;
    a.t_tiles = tiles_of(p.rows, size_of(h.logits).n);
    a.bias = p.bias;
    a.targets = targets;
    a.x_powers = h.split ? h.ranges.row : nullptr;
    a.w_powers = h.split ? h.ranges.entry : nullptr;
    a.scales = h.split && h.wants_dx ? h.scales : nullptr;
    return a;
}

// What both calls refuse.
static int refused(const dgs_head_args &p, bool back)
{
    if (p.cols == 0 || p.vocab == 0 || !is_type(p.type) || (p.target_bytes != 4 && p.target_bytes != 8)) return DGS_EINVAL;
    if (!matrix_ok(p.weight.data, p.weight.stride, p.cols, p.type) || !aligned_to(p.bias, 4)) return DGS_EINVAL;
    if (p.rows) {
        if (!matrix_ok(p.x.data, p.x.stride, p.cols, p.type) || !p.targets || !aligned_to(p.targets, p.target_bytes)) return DGS_EINVAL;
        if (!aligned_to(p.loss, 4) || !p.lse || !aligned_to(p.lse, 4)) return DGS_EINVAL;
        if (back && p.dx.data && !matrix_ok(p.dx.data, p.dx.stride, p.cols, p.type)) return DGS_EINVAL;
    }
    if (back && p.dweight && (p.dweight_stride < p.cols || p.dweight_stride >= (1ull << 32))) return DGS_EINVAL;
    if (!aligned_to(p.dloss, 4) || !aligned_to(p.dlse, 4) || !aligned_to(p.dweight, 4) || !aligned_to(p.dbias, 4)) return DGS_EINVAL;
    if (p.cols > (1u << 20) || p.rows > (1u << 24) || p.vocab > (1u << 24)) return DGS_ENOTSUP;
    // (a launch has less than 2^32 lanes: in tiles of 256 x 256, which products of that size take, a lane for 128 logits; a lane for eight values
    // of dx)
    if ((uint64_t)p.rows * p.vocab > (1ull << 38) || (uint64_t)p.rows * p.cols > (1ull << 34)) return DGS_ENOTSUP;
    return DGS_OK;
}

}  // namespace dgs

using namespace dgs;

extern "C" size_t dgs_head_workspace(const dgs_head_args *args, int backward)
{
    if (!args || refused(*args, backward != 0) != DGS_OK) return 0;
    return (size_t)plan_of(*args, backward != 0).bytes;
}

extern "C" int dgs_head_forward(const dgs_head_args *args, void *hip_stream)
{
    if (!args) return DGS_EINVAL;
    const dgs_head_args &p = *args;
    const int rc = refused(p, false);
    if (rc != DGS_OK) return rc;
    if (p.rows == 0) return DGS_OK;
    if (!p.workspace || !aligned_to(p.workspace, 16)) return DGS_EINVAL;
    const HeadPlan h = plan_of(p, false);
    if (p.workspace_bytes < h.bytes) return DGS_ENOMEM;
    if (p.loss && p.loss < p.lse + p.rows && p.lse < p.loss + p.rows) return DGS_EINVAL;      // (lse would be lost)
    const hipStream_t st = (hipStream_t)hip_stream;
    const Targets targets = {p.targets, p.target_bytes == 8, p.vocab};
    if (p.type == DGS_F32) prepare<float>(p, h, targets, st);
    else if (p.type == DGS_F16) prepare<f16>(p, h, targets, st);
    else prepare<bf16>(p, h, targets, st);
    LogitArgs a = logit_args(p, h, targets);
    a.end = p.vocab;
    a.v_tiles = tiles_of(p.vocab, size_of(h.logits).m);
    a.stats = h.stats;
    a.target_logit = h.target_logit;
    logits<false>(a, p.type, h.logits, st);
    const uint32_t apart = p.rows >= 2048 ? 8 : p.rows >= 64 ? 32 : 256;
    hipLaunchKernelGGL(k_head_loss, dim3(tiles_of(p.rows, 256 / apart)), dim3(256), 0, st, (const float2 *)h.stats,
                       (const float *)h.target_logit, targets, p.rows, a.v_tiles, apart, p.loss, p.lse);
    return launched();
}

extern "C" int dgs_head_backward(const dgs_head_args *args, void *hip_stream)
{
    if (!args) return DGS_EINVAL;
    const dgs_head_args &p = *args;
    const int rc = refused(p, true);
    if (rc != DGS_OK) return rc;
    if (p.rows == 0) {      // (no sums: zeros, or what is there)
        if (p.accumulate || (!p.dweight && !p.dbias)) return DGS_OK;
        if (p.dweight)
            hipLaunchKernelGGL(k_head_dweight, dim3(dweight_blocks(p.vocab, p.cols)), dim3(256), 0, (hipStream_t)hip_stream,
                               (const float *)nullptr, 0u, p.vocab, p.cols, (const Scales *)nullptr, p.dweight, p.dweight_stride, 0u);
        if (p.dbias)
            hipLaunchKernelGGL(k_head_dbias, dim3(tiles_of(p.vocab, 64)), dim3(256), 0, (hipStream_t)hip_stream,
                               BiasArgs{nullptr, 0, p.vocab, 0, 0, p.dbias});
        return launched();
    }
    if (!p.workspace || !aligned_to(p.workspace, 16)) return DGS_EINVAL;
    const HeadPlan h = plan_of(p, true);
    if (p.workspace_bytes < h.bytes) return DGS_ENOMEM;
    const hipStream_t st = (hipStream_t)hip_stream;
    const Targets targets = {p.targets, p.target_bytes == 8, p.vocab};
    const bool f32 = p.type == DGS_F32;
    if (p.type == DGS_F32) prepare<float>(p, h, targets, st);
    else if (p.type == DGS_F16) prepare<f16>(p, h, targets, st);
    else prepare<bf16>(p, h, targets, st);
    const TileSize tile = size_of(h.logits), tx = size_of(h.dx.tile), tw = size_of(h.dw.tile);
    const uint64_t stride = ((uint64_t)h.piece + 7) & ~7ull;
    const bool together = h.wants_dx && !h.few_dx && h.wants_dw && h.dx.tile == TILE_64 && h.dw.tile == TILE_64;
    LogitArgs a = logit_args(p, h, targets);
    a.row_info = h.row_info;
    a.grad[0] = h.grad[0];
    a.grad[1] = h.grad[1];
    a.grad_stride = stride;
    a.bias_parts = p.dbias ? h.bias_parts : nullptr;
    for (uint32_t first = 0; first < p.vocab; first += h.piece) {
        const uint32_t count = p.vocab - first < h.piece ? p.vocab - first : h.piece;
        a.first = first;
        a.end = first + count;
        a.v_tiles = tiles_of(count, tile.m);
        logits<true>(a, p.type, h.logits, st);
        const BiasArgs bias = {h.bias_parts, a.t_tiles, count, (uint32_t)(p.accumulate != 0), stride, p.dbias ? p.dbias + first : nullptr};
        if (p.dbias && !together) hipLaunchKernelGGL(k_head_dbias, dim3(tiles_of(count, 64)), dim3(256), 0, st, bias);
        GradientArgs dx = {};
        if (h.wants_dx && h.few_dx) {
            few_dx(p, h, first, count, stride, st);
        } else if (h.wants_dx) {
            GradientArgs &g = dx;
            const uint16_t *w = f32 ? h.w_all[0] : p.type == DGS_BF16 ? h.w[1] : h.copy_w ? h.w[0] : a.w.part[0];
            const uint64_t w_stride = p.type != DGS_F16 || h.copy_w ? h.width : a.w.stride;
            g.a = Side{{h.grad[0], h.grad[1]}, stride, p.rows};
            g.b = Side{{w + first * w_stride, f32 ? h.w_all[1] + first * w_stride : nullptr}, w_stride, p.cols};
            if (f32) {
                g.even[0] = h.w[0] + first * w_stride;
                g.even[1] = h.w[1] + first * w_stride;
                g.scales = h.scales;
            }
            g.depth = count;
            g.splits = h.dx.splits;
            g.split_depth = h.dx.split_depth;
            g.kind = h.dx.kind;
            g.m = p.rows;
            g.n = p.cols;
            g.m_tiles = tiles_of(g.m, tx.m);
            g.n_tiles = tiles_of(g.n, tx.n);
            g.out = h.dx_sums;
            g.out_stride = p.cols;
            g.add = first != 0;
            if (!together) product<false>(g, h.dx.tile, st);
        }
        if (h.wants_dw) {
            GradientArgs g = {};
            g.a = Side{{h.grad[0], h.grad[1]}, stride, count};
            g.b = Side{{h.x_weighed[0], h.x_weighed[1]}, h.width, p.cols};
            g.depth = p.rows;
            g.splits = h.dw.splits;
            g.split_depth = h.dw.split_depth;
            g.kind = h.dw.kind;
            g.m = count;
            g.n = p.cols;
            g.m_tiles = tiles_of(g.m, tw.m);
            g.n_tiles = tiles_of(g.n, tw.n);
            g.whole = g.splits == 1;
            g.out = g.whole ? p.dweight + first * p.dweight_stride : h.dw_sums;
            g.out_stride = g.whole ? p.dweight_stride : p.cols;
            g.add = g.whole && p.accumulate;
            g.scales = h.scales;
            if (together) {
                const uint32_t dw_blocks = g.m_tiles * g.n_tiles * g.splits, dx_blocks = dx.m_tiles * dx.n_tiles * dx.splits;
                hipLaunchKernelGGL(k_head_gradients, dim3(dw_blocks + dx_blocks + (p.dbias ? tiles_of(count, 64) : 0u)), dim3(256), 0, st, g, dx,
                                   bias, dw_blocks, dx_blocks);
            } else product<true>(g, h.dw.tile, st);
            if (h.dw.splits > 1)
                hipLaunchKernelGGL(k_head_dweight, dim3(dweight_blocks(count, p.cols)), dim3(256), 0, st,
                                   (const float *)h.dw_sums, g.splits, count, p.cols, (const Scales *)h.scales,
                                   p.dweight + first * p.dweight_stride, p.dweight_stride, (uint32_t)(p.accumulate != 0));
        }
    }
    if (h.wants_dx) {
        const Scales *const sc = h.scale_w ? h.scales : nullptr;
        if (f32) finish_dx<float>(p, h, sc, st);
        else if (p.type == DGS_F16) finish_dx<f16>(p, h, sc, st);
        else finish_dx<bf16>(p, h, sc, st);
    }
    return launched();
}
