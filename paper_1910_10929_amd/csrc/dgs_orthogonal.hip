// Updates orthogonalised by Newton-Schulz products: X = G / (|G| + eps), then `steps` times with A = X X^T
//
//     X = a X + (b A + c A^2) X
//
// which leaves G's singular vectors and takes its singular values towards 1 (X^T in place of X where rows outnumber columns, so
// that A is the smaller square).  Matrices of up to 128 x 128 take one launch, others three a step: the two symmetric products, of which tiles on and below the diagonal
// are computed and stored twice, and the product with X.
//
// Numbers.  Sums are fp32, the norm's in 64 bits.  Between the products X is held in two halves (22 bits), times 2^12.  The
// polynomial B = a I + b A + c A^2 is held without its diagonal, which stays in fp32 and meets X in the last product's epilogue:
// most of what B does to X is its diagonal, and half's rounding of the rest is small beside it.  Results in bfloat16 take the
// first half of each operand to the products; half and fp32 results take both, and A and B are held in two halves then.
#include "dgs_product.h"

namespace dgs {

constexpr float HELD = 4096.0f, LEFT = 1.0f / HELD;      // X, A and B are held times 2^12
constexpr uint32_t ORTHO_AT_ONCE = 32;      // matrices of a launch
constexpr uint32_t NORM_PARTS = 256;      // at most
#ifdef DGS_HOST_EMULATION
constexpr uint32_t SMALL = 1u << 10;
#else
constexpr uint32_t SMALL = 1u << 14;      // values of a matrix whose norm has no launch of its own (2^14 of them: 6.2 us, in two launches 3.6 and 4.2)
#endif

struct Matrices {
    const void *data[ORTHO_AT_ONCE];
    uint64_t stride[ORTHO_AT_ONCE];
};
struct Halves {
    uint16_t *hi, *lo;
    uint64_t stride, size;      // from row to row, and of a matrix
};

// An update whose norm is far below eps starts with an X far below 1.  X is then held times 2^lift besides, so that what half's
// smallest numbers cut off stays as far below it as ever.  The lift follows a bound on X's singular values, here its log2: the norm at the
// start, and a step takes s to at most s (|a| + |b| s^2 + |c| s^4).  (Not |a|^step: with |a| < 1 that goes to 0 where b and c keep singular
// values near 1.)
__device__ __forceinline__ int lift_of(float bound)
{
    return bound <= -1.0f ? (int)min(-bound, 120.0f) : 0;      // (a NaN: 0)
}
struct Coefficients { float a, b, c; };
__device__ __forceinline__ float bound_after(float bound, const Coefficients &by)
{
    const float square = exp2f(2.0f * bound);
    return bound + log2f(__builtin_fabsf(by.a) + (__builtin_fabsf(by.b) + __builtin_fabsf(by.c) * square) * square);
}
__device__ __forceinline__ float times_power(float v, int e)
{
#ifdef DGS_HOST_EMULATION
    return ldexpf(v, e);
#else
    return __builtin_amdgcn_ldexpf(v, e);
#endif
}
__device__ __forceinline__ void put_halves(const Halves &to, uint64_t at, const float (&v)[8])
{
    u32x4 hi, lo;
    halves8(v, hi, lo);
    *(u32x4 *)(to.hi + at) = hi;
    if (to.lo) *(u32x4 *)(to.lo + at) = lo;
}

// A lane's sum of squares: of eight columns at a time, from the `at`-th eight on, `step` further each turn.
template <class T> __device__ __forceinline__ double squares(const T *m, uint64_t stride, uint32_t rows, uint32_t cols, uint32_t at, uint32_t step)
{
    const uint32_t pieces = (cols + 7) / 8, end = pieces * rows;      // (at most 2^29)
    double s = 0.0;
    for (; at < end; at += step) {
        const uint32_t row = at / pieces, c = (at - row * pieces) * 8;
        float v[8];
        unpack8(load8(m + row * stride + c, live8(c, cols)), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += (double)v[i] * (double)v[i];
    }
    return s;
}

// Sums of squares, at most NORM_PARTS a matrix.  Bound by memory: twelve of 2304 x 768 in fp32, 85 MB, 16.4 us (5.2 TB/s).
template <class T>
__global__ __launch_bounds__(256) void k_ortho_norm(Matrices in, uint32_t rows, uint32_t cols, double *parts)
{
    __shared__ double sums[256];
    const uint32_t which = blockIdx.y;
    sums[threadIdx.x] = squares((const T *)in.data[which], in.stride[which], rows, cols, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
    __syncthreads();
    for (uint32_t by = 128; by; by >>= 1) {
        if (threadIdx.x < by) sums[threadIdx.x] += sums[threadIdx.x + by];
        __syncthreads();
    }
    if (threadIdx.x == 0) parts[which * gridDim.x + blockIdx.x] = sums[0];
}

// X from G, 64 x 64 of it to a workgroup, turned where that makes it wide.  Columns up to a multiple of eight are zeros.
// Bound by memory: twelve of 2304 x 768, 85 MB read and as many written, 34 us (5.0 TB/s).  norm_parts = 0: every workgroup takes the norm
// of its matrix itself.
template <class T>
__global__ __launch_bounds__(256) void k_ortho_load(Matrices in, uint32_t rows, uint32_t cols, uint32_t turned, const double *parts, uint32_t norm_parts,
                                                    float eps, Halves x, float *bound)
{
    __shared__ double norm[NORM_PARTS];
    __shared__ float tile[64][65];
    const uint32_t which = blockIdx.y, across = (cols + 63) / 64;
    const T *const m = (const T *)in.data[which];
    const uint64_t stride = in.stride[which];
    if (norm_parts == 0) norm[threadIdx.x] = squares(m, stride, rows, cols, threadIdx.x, NORM_PARTS);
    else norm[threadIdx.x] = threadIdx.x < norm_parts ? parts[which * norm_parts + threadIdx.x] : 0.0;
    for (uint32_t by = NORM_PARTS / 2; by; by >>= 1) {
        __syncthreads();
        if (threadIdx.x < by) norm[threadIdx.x] += norm[threadIdx.x + by];
    }
    __syncthreads();
    const double sum = norm[0];
    const double length = sqrt(sum), whole = length + (double)eps;
    const float log2_of = sum > 0.0 ? (float)(log2(length) - log2(whole)) : 0.0f;
    const double by = ldexp((double)HELD, lift_of(log2_of)) / whole;
    if (blockIdx.x == 0 && threadIdx.x == 0) bound[which] = log2_of;
    const uint32_t r0 = blockIdx.x / across * 64, c0 = blockIdx.x % across * 64;      // of G
    const uint32_t c = (threadIdx.x & 7u) * 8, n = live8(c0 + c, cols);
    Raw8<T> raw[2];
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t r = r0 + 32 * i + (threadIdx.x >> 3);
        raw[i] = load8(m + (r < rows && n ? r * stride + c0 + c : 0u), r < rows ? n : 0u);
    }
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        float v[8];
        unpack8(raw[i], v);
#pragma unroll
        for (int k = 0; k < 8; ++k) tile[32 * i + (threadIdx.x >> 3)][c + k] = (float)((double)v[k] * by);
    }
    __syncthreads();
    const uint32_t x_rows = turned ? cols : rows;
    const uint32_t first_row = turned ? c0 : r0, first_col = turned ? r0 : c0;
#pragma unroll
    for (uint32_t at = threadIdx.x; at < 64 * 8; at += 256) {
        const uint32_t i = at >> 3, q = (at & 7u) * 8;
        if (first_row + i >= x_rows || first_col + q >= x.stride) continue;
        float v[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) v[k] = turned ? tile[q + k][i] : tile[i][q + k];
        put_halves(x, which * x.size + (first_row + i) * x.stride + first_col + q, v);
    }
}

struct SquareArgs {
    Halves x;                // both operands: rows of it by rows of it
    uint32_t depth, kind;
    uint32_t size, tiles;    // of the result, and tiles along a side
    uint32_t count;          // matrices
    uint32_t split_depth;    // of a split of the sum; as long as it is for a single one
    float *sums;             // with several: size x out.stride for each split and matrix, on and below the diagonal
    const float *bound;      // of each X; absent: nothing was lifted
    Halves out;              // lo: absent where products take the first halves
    // the polynomial: b A + c A^2, and its diagonal
    Halves gram;
    float *diagonal;         // size a matrix
    Coefficients by;
};

// What becomes of a row's eight sums from column n on: A, or the polynomial without its diagonal.
template <bool POLY>
__device__ __forceinline__ void finish8(const SquareArgs &a, uint32_t which, uint32_t m, uint32_t n, int power, const u32x4 &gram_hi,
                                        const u32x4 &gram_lo, float (&v)[8])
{
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
        v[k] = times_power(v[k], power);
        if constexpr (POLY) {
            const float gram = half_value((uint16_t)(gram_hi[k >> 1] >> (16 * (k & 1)))) + half_value((uint16_t)(gram_lo[k >> 1] >> (16 * (k & 1))));
            v[k] = a.by.b * gram + a.by.c * v[k];
        }
    }
    if constexpr (POLY) {
        if (n <= m && m < n + 8) {
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
                if (n + k == m) {
                    if (m < a.size) a.diagonal[which * a.size + m] = a.by.a + v[k] * LEFT;
                    v[k] = 0.0f;
                }
        }
    }
}
// A's row m, columns n to n + 7.
__device__ __forceinline__ void gram8(const SquareArgs &a, uint64_t from, uint32_t m, uint32_t n, u32x4 &hi, u32x4 &lo)
{
    const u32x4 none = {0, 0, 0, 0};
    hi = lo = none;
    if (m < a.size && n < a.gram.stride) {
        hi = *(const u32x4 *)(a.gram.hi + from + m * a.gram.stride + n);
        if (a.gram.lo) lo = *(const u32x4 *)(a.gram.lo + from + m * a.gram.stride + n);
    }
}
__device__ __forceinline__ int power_of_sums(const SquareArgs &a, uint32_t which)
{
    return -12 - (a.bound ? 2 * lift_of(a.bound[which]) : 0);
}

// The symmetric product of X with itself (POLY: of A with itself, from which the polynomial is made).  Bound by the matrix units:
// 4096 x 4096 (69 GFLOP of tiles) 78 and 84 us, 192 x 192 so that 253 of 256 compute units have one tile each; 256 x 256, 136 tiles, takes 93
// and 94, 128 x 128 107 and 111.  333 x 1001 (five, three pairs): by latency, 48 steps of 64 x 64 in 17 us.
template <uint32_t M, uint32_t WAVES_M, uint32_t WAVES_N, uint32_t STAGES, bool POLY>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64, M == 192 ? 1 : 2) void k_ortho_square(SquareArgs a)
{
    typedef Product<f16, M, M, WAVES_M, WAVES_N, false, false, STAGES> P;
    __shared__ __attribute__((aligned(16))) typename P::Lds lds;
    // tiles on and below the diagonal, row by row
    const uint32_t count = a.tiles * (a.tiles + 1) / 2;
    const uint32_t all = tile_of_block(blockIdx.x, gridDim.x), each = all / count, at = all - each * count;
    const uint32_t split = each / a.count, which = each - split * a.count;
    uint32_t tile_m = 0, passed = 0;
    while (passed + tile_m + 1 <= at) passed += ++tile_m;
    const uint32_t tile_n = at - passed;
    const Side side = {{a.x.hi + which * a.x.size, a.x.lo ? a.x.lo + which * a.x.size : nullptr}, a.x.stride, a.size};
    const uint32_t first = split * a.split_depth;
    const uint64_t base = which * a.out.size, from = which * a.gram.size;
    u32x4 gram_hi[P::PASSES], gram_lo[P::PASSES];
    auto look = [&](uint32_t p, uint32_t row, uint32_t col) {
        if constexpr (POLY) gram8(a, from, tile_m * M + row, tile_n * M + col, gram_hi[p], gram_lo[p]);
    };
    P::look_early(look);
    typename P::Sums s;
    P::run(lds, side, side, tile_m * M, tile_n * M, first, min(first + a.split_depth, a.depth), a.kind, s);
    if (a.sums) {
        float *const sums = a.sums + (uint64_t)each * a.size * a.out.stride;
        P::by_rows(lds, s, [&](uint32_t, uint32_t, uint32_t) {}, [&](uint32_t, uint32_t row, uint32_t col, float (&v)[8]) {
            const uint32_t m = tile_m * M + row, n = tile_n * M + col;
            if (m >= a.size || n >= a.out.stride) return;
            f32x4 w;
            w.x = v[0]; w.y = v[1]; w.z = v[2]; w.w = v[3];
            *(f32x4 *)(sums + m * a.out.stride + n) = w;
            w.x = v[4]; w.y = v[5]; w.z = v[6]; w.w = v[7];
            *(f32x4 *)(sums + m * a.out.stride + n + 4) = w;
        });
        return;
    }
    const int power = power_of_sums(a, which);
    // (the result's columns are a multiple of eight, those beyond its rows zeros)
    P::by_rows(lds, s, look, [&](uint32_t p, uint32_t row, uint32_t col, float (&v)[8], float *back) {
        const uint32_t m = tile_m * M + row, n = tile_n * M + col;
        finish8<POLY>(a, which, m, n, power, gram_hi[p], gram_lo[p], v);
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) back[k] = v[k];
        if (m < a.size && n < a.out.stride) put_halves(a.out, base + m * a.out.stride + n, v);
    }, [&](uint32_t row, uint32_t col, const float (&v)[8]) {      // the other side of the diagonal
        const uint32_t m = tile_m * M + row, n = tile_n * M + col;
        if (tile_m != tile_n && n < a.size && m < a.out.stride) put_halves(a.out, base + n * a.out.stride + m, v);
    });
}

// The same from several splits' sums: 64 x 64 of the result, on or below the diagonal, to a workgroup.
template <bool POLY> __global__ __launch_bounds__(256) void k_ortho_join(SquareArgs a, uint32_t splits, uint32_t tiles)
{
    __shared__ float turned[64][65];
    const uint32_t count = tiles * (tiles + 1) / 2;
    const uint32_t which = blockIdx.x / count, at = blockIdx.x - which * count;
    uint32_t tile_m = 0, passed = 0;
    while (passed + tile_m + 1 <= at) passed += ++tile_m;
    const uint32_t tile_n = at - passed;
    const uint64_t base = which * a.out.size, from = which * a.gram.size, apart = (uint64_t)a.count * a.size * a.out.stride;
    const int power = power_of_sums(a, which);
    const uint32_t c = (threadIdx.x & 7u) * 8, n = tile_n * 64 + c;
    const bool column = n < a.out.stride;
#pragma unroll
    for (uint32_t i = 0; i < 64; i += 32) {
        const uint32_t r = i + (threadIdx.x >> 3), m = tile_m * 64 + r;
        float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        u32x4 hi = {0, 0, 0, 0}, lo = hi;
        if constexpr (POLY) gram8(a, from, m, n, hi, lo);
        if (m < a.size && column) {
            const float *const p = a.sums + ((uint64_t)which * a.size + m) * a.out.stride + n;
            for (uint32_t s = 0; s < splits; ++s) {
                const f32x4 x = *(const f32x4 *)(p + s * apart), y = *(const f32x4 *)(p + s * apart + 4);
                v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
            }
            finish8<POLY>(a, which, m, n, power, hi, lo, v);
            put_halves(a.out, base + m * a.out.stride + n, v);
        }
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) turned[r][c + k] = v[k];
    }
    __syncthreads();
    if (tile_m == tile_n) return;
#pragma unroll
    for (uint32_t i = 0; i < 64; i += 32) {
        const uint32_t r = i + (threadIdx.x >> 3), row = tile_n * 64 + r, col = tile_m * 64 + c;
        if (row >= a.size || col >= a.out.stride) continue;
        float v[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) v[k] = turned[c + k][r];
        put_halves(a.out, base + row * a.out.stride + col, v);
    }
}

struct StepArgs {
    Halves poly, x, next;      // next.hi: absent in the last step
    const float *diagonal;
    uint32_t rows, cols, kind;
    uint32_t m_tiles, n_tiles;
    const float *bound;      // of each X, and (but in the last step) of its next
    float *next_bound;
    Coefficients by;
    // the last step
    uint32_t add;
    float scale;
};

template <class T> __device__ __forceinline__ void put8(T *p, uint32_t count, float (&v)[8], float scale, uint32_t add)
{
    float old[8];
    if (add) unpack8(load8((const T *)p, count), old);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = add ? old[k] + v[k] * scale : v[k] * scale;
    store8(p, 0, count, v);
}

// X of the next step: its rows times the polynomial's diagonal, plus the product of the rest with it.  4096 x 4096: 132 us (1040 TFLOP/s
// with one round of tiles); twelve of 768 x 2304: 62 us, 212 MB of X's halves read twice over and written beside 33 GFLOP.
// T: the result's type in the last step, void in the others; TURNED: the result's rows are X's columns.
template <uint32_t M, uint32_t WAVES_M, uint32_t WAVES_N, uint32_t STAGES, class T, bool TURNED>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64, 2) void k_ortho_step(StepArgs a, Matrices results)
{
    typedef Product<f16, M, M, WAVES_M, WAVES_N, false, true, STAGES> P;
    __shared__ __attribute__((aligned(16))) typename P::Lds lds;
    const uint32_t count = a.m_tiles * a.n_tiles;
    const uint32_t all = tile_of_block(blockIdx.x, gridDim.x), which = all / count, at = all - which * count;
    const TilePlace place = place_of_tile(at, a.m_tiles, a.n_tiles);
    const uint32_t tile_m = place.m, tile_n = place.n;
    const uint16_t *const x_hi = a.x.hi + which * a.x.size, *const x_lo = a.x.lo + which * a.x.size;
    const Side left = {{a.poly.hi + which * a.poly.size, a.poly.lo ? a.poly.lo + which * a.poly.size : nullptr}, a.poly.stride, a.rows};
    const Side right = {{x_hi, x_lo}, a.x.stride, a.cols};
    // a row of X's next, or of the result's
    u32x4 hi[P::PASSES], lo[P::PASSES];
    float d[P::PASSES];
    auto look = [&](uint32_t p, uint32_t row, uint32_t col) {
        const uint32_t m = tile_m * M + row, n = tile_n * M + col;
        const bool in = m < a.rows && n < a.x.stride;
        const uint64_t at = in ? m * a.x.stride + n : 0;
        hi[p] = *(const u32x4 *)(x_hi + at);
        lo[p] = *(const u32x4 *)(x_lo + at);
        d[p] = a.diagonal[which * a.rows + (in ? m : 0)];
    };
    P::look_early(look);
    typename P::Sums s;
    P::run(lds, left, right, tile_m * M, tile_n * M, 0, a.rows, a.kind, s);
    // from how this X is held to how the next one is, or to the result
    const float bound = a.bound[which];
    const int lift = lift_of(bound);
    int power = -12 - lift;
    if constexpr (__is_same(T, void)) {
        const float next_bound = bound_after(bound, a.by);
        power = lift_of(next_bound) - lift;
        if (at == 0 && threadIdx.x == 0) a.next_bound[which] = next_bound;
    }
    auto next = [&](uint32_t p, float (&v)[8]) {
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
            const float x = half_value((uint16_t)(hi[p][k >> 1] >> (16 * (k & 1)))) + half_value((uint16_t)(lo[p][k >> 1] >> (16 * (k & 1))));
            v[k] = times_power(__builtin_fmaf(d[p], x, v[k] * LEFT), power);
        }
    };
    if constexpr (__is_same(T, void)) {
        P::by_rows(lds, s, look, [&](uint32_t p, uint32_t row, uint32_t col, float (&v)[8]) {
            const uint32_t m = tile_m * M + row, n = tile_n * M + col;
            next(p, v);
            if (m < a.rows && n < a.x.stride) put_halves(a.next, which * a.next.size + m * a.x.stride + n, v);
        });
    } else {
        T *const out = (T *)results.data[which];
        const uint64_t stride = results.stride[which];
        if constexpr (TURNED) {
            P::by_rows(lds, s, look, [&](uint32_t p, uint32_t, uint32_t, float (&v)[8], float *back) {
                next(p, v);
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) back[k] = v[k];
            }, [&](uint32_t row, uint32_t col, float (&v)[8]) {
                const uint32_t m = tile_m * M + row, n = tile_n * M + col;
                if (m < a.rows && n < a.cols) put8(out + n * stride + m, live8(m, a.rows), v, a.scale, a.add);
            });
        } else {
            P::by_rows(lds, s, look, [&](uint32_t p, uint32_t row, uint32_t col, float (&v)[8]) {
                const uint32_t m = tile_m * M + row, n = tile_n * M + col;
                next(p, v);
                if (m < a.rows && n < a.cols) put8(out + m * stride + n, live8(n, a.cols), v, a.scale, a.add);
            });
        }
    }
}

// Matrices of up to S x S, whole: a workgroup each, all steps in one launch.  A lane keeps its values of X and A in fp32; what the products
// read of them lies in LDS in halves, transposed, so that the four rows that a lane has together are written together (A and the polynomial are
// symmetric).  Bound by latency: of 128 x 128 a product is 24 matrix instructions a wavefront between two barriers (eight slices, three pairs of parts), each
// of two fragments from LDS, 768 KB in all: some 2.6 us of the 4.8 that a product takes.  A square of 32 x 32 to a wavefront, so that
// four of them share a SIMD at 128 x 128: five steps of one in fp32 73 us (four wavefronts with four squares each: 102; in launches of their own, 16 of
// them: 98); 64 x 64 31 (81); 32 of 128 x 128 in bfloat16 46 (89); 200 of 48 x 48 in fp32 245 (563).
struct SmallArgs {
    uint32_t rows, cols, turned, type, out_type;      // of G
    uint32_t steps, kind, add;
    Coefficients by;
    float eps, scale;
};
__device__ __forceinline__ float value_at(const void *p, uint64_t at, uint32_t type)
{
    return type == DGS_F32 ? ((const float *)p)[at] : type == DGS_F16 ? to_float(((const f16 *)p)[at]) : to_float(((const bf16 *)p)[at]);
}
__device__ __forceinline__ void put_value(void *p, uint64_t at, uint32_t type, float v)
{
    if (type == DGS_F32) ((float *)p)[at] = v;
    else if (type == DGS_F16) ((f16 *)p)[at] = from_float<f16>(v);
    else ((bf16 *)p)[at] = from_float<bf16>(v);
}
template <uint32_t S> struct Small {
    static constexpr uint32_t SIDE = S / 32, THREADS = SIDE * SIDE * 64, PITCH = S + 8;      // (4 banks more than a multiple of 32)
    typedef uint16_t Part[S][PITCH];

    // A wavefront has a square of 32 x 32.
    static __device__ __forceinline__ uint32_t wave_m() { return uniform(threadIdx.x >> 6) / SIDE * 32; }
    static __device__ __forceinline__ uint32_t wave_n() { return uniform(threadIdx.x >> 6) % SIDE * 32; }

    // Values as halves, transposed; `two`: what the first half leaves, too.
    static __device__ __forceinline__ void put(Part *to, const f32x16 &v, bool two)
    {
        const uint32_t n = wave_n() + (lane_id() & 31u);
#pragma unroll
        for (uint32_t g = 0; g < 4; ++g) {
            const uint32_t m = wave_m() + square_row(4 * g);
            u32x2 hi, lo;
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
                const f32x2 w = {v[4 * g + 2 * k], v[4 * g + 2 * k + 1]};
                const f16x2 h = __builtin_convertvector(w, f16x2);
                const f32x2 left = {w.x - (float)h.x, w.y - (float)h.y};
                hi[k] = __builtin_bit_cast(uint32_t, h);
                lo[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(left, f16x2));
            }
            *(u32x2 *)&to[0][n][m] = hi;
            if (two) *(u32x2 *)&to[1][n][m] = lo;
        }
    }
    // 32 rows from `first` on of an operand, k from 16 s on: k inside (TURNED: outside).
    template <bool TURNED> static __device__ __forceinline__ u32x4 fragment(const Part &p, uint32_t first, uint32_t s)
    {
        const uint32_t lane = lane_id();
        if constexpr (!TURNED) return *(const u32x4 *)&p[first + (lane & 31u)][16 * s + 8 * (lane >> 5)];
        const uint32_t k = 16 * s + ((lane >> 5) << 3) + ((lane & 15u) >> 2), c = first + ((lane >> 4) & 1u) * 16 + (lane & 3u) * 4;
        const u32x2 x = read_turned(&p[k][c]), y = read_turned(&p[k + 4][c]);
        return u32x4{x.x, x.y, y.x, y.y};
    }
    template <bool TURNED> static __device__ __forceinline__ f32x16 product(const Part *a, const Part *b, uint32_t depth, uint32_t kind)
    {
        f32x16 c;
#pragma unroll
        for (uint32_t r = 0; r < 16; ++r) c[r] = 0.0f;
        const uint32_t slices = (depth + 15) / 16;
        for (uint32_t pair = 0; pair < pairs_of(kind); ++pair) {
            const Part &pa = a[pair == 1], &pb = b[pair == 2];
#pragma unroll 4
            for (uint32_t s = 0; s < slices; ++s)
                c = matrix_unit_of<f16>(fragment<TURNED>(pa, wave_m(), s), fragment<TURNED>(pb, wave_n(), s), c);
        }
        return c;
    }
};
template <uint32_t S> __global__ __launch_bounds__(Small<S>::THREADS, 1) void k_ortho_small(SmallArgs a, Matrices in, Matrices results)
{
    typedef Small<S> P;
    __shared__ __attribute__((aligned(16))) typename P::Part x_lds[2], square[2];
    __shared__ float diagonal[S];
    __shared__ double norm[P::THREADS];
    const uint32_t which = blockIdx.x;
    const uint32_t x_rows = a.turned ? a.cols : a.rows, x_cols = a.turned ? a.rows : a.cols;
    const bool two = a.kind != ONE_PAIR;
    // this lane's column, and its rows, of X; rows 4 g to 4 g + 3 of its sixteen lie together
    const uint32_t n = P::wave_n() + (lane_id() & 31u);
    uint32_t m[16];
#pragma unroll
    for (uint32_t r = 0; r < 16; ++r) m[r] = P::wave_m() + square_row(r);
    f32x16 x, v, gram;
    const void *const from = in.data[which];
    const uint64_t stride = in.stride[which];
    double sum = 0.0;
#pragma unroll
    for (uint32_t r = 0; r < 16; ++r) {
        const bool here = m[r] < x_rows && n < x_cols;
        x[r] = here ? value_at(from, a.turned ? n * stride + m[r] : m[r] * stride + n, a.type) : 0.0f;
        sum += (double)x[r] * (double)x[r];
    }
    norm[threadIdx.x] = sum;
    for (uint32_t by = P::THREADS / 2; by; by >>= 1) {
        __syncthreads();
        if (threadIdx.x < by) norm[threadIdx.x] += norm[threadIdx.x + by];
    }
    __syncthreads();
    const double length = sqrt(norm[0]), whole = length + (double)a.eps;
    float bound = norm[0] > 0.0 ? (float)(log2(length) - log2(whole)) : 0.0f;
    int lift = lift_of(bound);
    const double by = ldexp((double)HELD, lift) / whole;
#pragma unroll
    for (uint32_t r = 0; r < 16; ++r) x[r] = m[r] < x_rows && n < x_cols ? (float)((double)x[r] * by) : 0.0f;
    for (uint32_t step = 0; step < a.steps; ++step) {
        P::put(x_lds, x, two);
        __syncthreads();
        gram = P::template product<true>(x_lds, x_lds, x_cols, a.kind);
        // (A as the products read it, in the polynomial too: near 1 what its rounding does to b A and c A^2 cancels but for a fifth)
#pragma unroll
        for (uint32_t r = 0; r < 16; ++r) {
            gram[r] = times_power(gram[r], -12 - 2 * lift);
            if (!two) gram[r] = to_float(from_float<f16>(gram[r]));
        }
        P::put(square, gram, two);
        __syncthreads();
        v = P::template product<false>(square, square, x_rows, a.kind);
        __syncthreads();      // (A has been read)
#pragma unroll
        for (uint32_t r = 0; r < 16; ++r) {
            v[r] = a.by.b * gram[r] + a.by.c * times_power(v[r], -12);
            if (m[r] == n) {
                diagonal[n] = a.by.a + v[r] * LEFT;
                v[r] = 0.0f;
            }
        }
        P::put(square, v, two);
        __syncthreads();
        v = P::template product<false>(square, x_lds, x_rows, a.kind);
        bound = bound_after(bound, a.by);
        const int next_lift = step + 1 < a.steps ? lift_of(bound) : -12;
#pragma unroll
        for (uint32_t r = 0; r < 16; ++r) x[r] = times_power(__builtin_fmaf(diagonal[m[r]], x[r], v[r] * LEFT), next_lift - lift);
        lift = next_lift;
        __syncthreads();      // (X and the polynomial have been read)
    }
    if (n >= x_cols) return;
    void *const to = (void *)results.data[which];
    const uint64_t out_stride = results.stride[which];
#pragma unroll
    for (uint32_t r = 0; r < 16; ++r) {
        if (m[r] >= x_rows) continue;
        const uint64_t at = a.turned ? n * out_stride + m[r] : m[r] * out_stride + n;
        put_value(to, at, a.out_type, a.add ? value_at(to, at, a.out_type) + x[r] * a.scale : x[r] * a.scale);
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

// A symmetric product's tile, and how many splits of its sum another launch adds up.
struct SquarePlan {
    int tile;
    uint32_t splits, split_depth;
};
static SquarePlan square_plan(uint32_t size, uint32_t depth, uint32_t pairs, uint32_t count)
{
    SquarePlan best = {};
    float least = 0.0f;
    const uint32_t steps = tiles_of(depth, PRODUCT_STEP), most = splits_tried(steps, 8);
    for (uint32_t s = 1; s <= most; ++s) {
        const uint32_t each = (steps + s - 1) / s;
        if ((steps + each - 1) / each != s) continue;
        float us = 0.0f;
        const int tile = product_tile([=](uint32_t high, uint32_t) { const uint64_t t = tiles_of(size, high); return t * (t + 1) / 2 * count * s; },
                                      each * pairs, TILE_192, us);
        // (the sums of half the square and more are written and read)
        if (s > 1) us += 6.0f + (float)s * (float)count * (float)size * (float)size * 5.0f / 4.5e6f;
        if (least == 0.0f || us < least || MOST_SPLITS) {
            least = us;
            best = SquarePlan{tile, s, each * PRODUCT_STEP};
        }
    }
    return best;
}
// Matrices up to this side take one launch for all of their steps.  (A CPU build that splits products is there for the others.)
#ifdef DGS_PRODUCT_SPLITS
constexpr uint32_t SMALL_SIDE = 0;
#else
constexpr uint32_t SMALL_SIDE = 128;
#endif
struct OrthoPlan {
    uint32_t rows, cols, at_once;      // of X, and matrices of a launch
    bool turned, two;
    Halves x[2], gram, poly;
    double *norm;
    float *diagonal, *bound[2], *sums;      // (bound: of a step's X, and of the next one's)
    SquarePlan square, poly_square;      // of X with itself, of A with itself
    uint64_t bytes;
};
static OrthoPlan ortho_plan(const dgs_orthogonalise_args &p)
{
    OrthoPlan o = {};
    o.turned = p.rows > p.cols;
    o.rows = o.turned ? p.cols : p.rows;
    o.cols = o.turned ? p.rows : p.cols;
    o.two = p.out_type != DGS_BF16;
    const uint64_t wide = (o.cols + 7ull) & ~7ull, small = (o.rows + 7ull) & ~7ull;
    uint64_t most = (1ull << 28) / (wide * o.rows);      // (values of X at a time: enough to fill the chip)
    if (most > ORTHO_AT_ONCE) most = ORTHO_AT_ONCE;
    if (most < 1) most = 1;
    o.at_once = most < p.count ? (uint32_t)most : p.count;
    Sections s = {(uintptr_t)p.workspace, 0};
    auto halves = [&](uint64_t stride, uint64_t rows, bool lo) {
        Halves h = {nullptr, nullptr, stride, stride * rows};
        h.hi = (uint16_t *)s.take(h.size * o.at_once * 2);
        if (lo) h.lo = (uint16_t *)s.take(h.size * o.at_once * 2);
        return h;
    };
    o.x[0] = halves(wide, o.rows, true);
    o.x[1] = halves(wide, o.rows, true);
    o.gram = halves(small, o.rows, o.two);
    o.poly = halves(small, o.rows, o.two);
    o.norm = (double *)s.take(sizeof(double) * NORM_PARTS * o.at_once);
    o.diagonal = (float *)s.take(4ull * o.rows * o.at_once);
    for (float *&b : o.bound) b = (float *)s.take(4ull * o.at_once);
    o.square = square_plan(o.rows, o.cols, o.two ? 3 : 1, o.at_once);
    o.poly_square = square_plan(o.rows, o.rows, o.two ? 3 : 1, o.at_once);
    const uint32_t splits = o.square.splits > o.poly_square.splits ? o.square.splits : o.poly_square.splits;
    if (splits > 1) o.sums = (float *)s.take(4ull * splits * o.at_once * o.rows * small);
    o.bytes = s.used;
    return o;
}

static int ortho_refused(const dgs_orthogonalise_args &p)
{
    if (p.rows == 0 || p.cols == 0 || p.steps == 0 || !is_type(p.type) || !is_type(p.out_type) || !(p.eps >= 0.0f)) return DGS_EINVAL;
    if (p.rows > (1u << 16) || p.cols > (1u << 16)) return DGS_ENOTSUP;
    return DGS_OK;
}

template <class T> static void load_matrices(const Matrices &in, const dgs_orthogonalise_args &p, const OrthoPlan &o, uint32_t count, hipStream_t st)
{
    // (a workgroup for every 64 KB or so of halves, and as few as there are work)
    const uint64_t work = (uint64_t)p.rows * ((p.cols + 7) / 8) / 2048 + 1;
    const uint32_t parts = (uint64_t)p.rows * p.cols <= SMALL ? 0u : work < NORM_PARTS ? (uint32_t)work : NORM_PARTS;
    if (parts) hipLaunchKernelGGL(k_ortho_norm<T>, dim3(parts, count), dim3(256), 0, st, in, p.rows, p.cols, o.norm);
    hipLaunchKernelGGL(k_ortho_load<T>, dim3((p.cols + 63) / 64 * ((p.rows + 63) / 64), count), dim3(256), 0, st, in, p.rows, p.cols,
                       (uint32_t)o.turned, (const double *)o.norm, parts, p.eps, o.x[0], o.bound[0]);
}

template <class T, bool TURNED> static void launch_step(const StepArgs &s, const Matrices &out, int tile, uint32_t count, hipStream_t st)
{
    const dim3 grid(s.m_tiles * s.n_tiles * count);
    if (tile == TILE_256) hipLaunchKernelGGL((k_ortho_step<256, 2, 4, 2, T, TURNED>), grid, dim3(512), 0, st, s, out);
    else if (tile == TILE_128) hipLaunchKernelGGL((k_ortho_step<128, 2, 2, 2, T, TURNED>), grid, dim3(256), 0, st, s, out);
    else hipLaunchKernelGGL((k_ortho_step<64, 2, 2, 4, T, TURNED>), grid, dim3(256), 0, st, s, out);
}
template <bool POLY> static void launch_square(SquareArgs a, const SquarePlan &plan, float *sums, hipStream_t st)
{
    a.tiles = tiles_of(a.size, tile_high(plan.tile));
    a.split_depth = plan.split_depth;
    a.sums = plan.splits > 1 ? sums : nullptr;
    const int tile = plan.tile;
    const dim3 grid(a.tiles * (a.tiles + 1) / 2 * a.count * plan.splits);
    if (tile == TILE_256) hipLaunchKernelGGL((k_ortho_square<256, 2, 4, 2, POLY>), grid, dim3(512), 0, st, a);
    else if (tile == TILE_192) hipLaunchKernelGGL((k_ortho_square<192, 2, 2, 2, POLY>), grid, dim3(256), 0, st, a);
    else if (tile == TILE_128) hipLaunchKernelGGL((k_ortho_square<128, 2, 2, 2, POLY>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_ortho_square<64, 2, 2, 4, POLY>), grid, dim3(256), 0, st, a);
    if (plan.splits > 1) {
        const uint32_t tiles = tiles_of(a.size, 64);
        hipLaunchKernelGGL(k_ortho_join<POLY>, dim3(tiles * (tiles + 1) / 2 * a.count), dim3(256), 0, st, a, plan.splits, tiles);
    }
}
template <class T> static void launch_last(const StepArgs &s, const Matrices &out, bool turned, int tile, uint32_t count, hipStream_t st)
{
    if (turned) launch_step<T, true>(s, out, tile, count, st);
    else launch_step<T, false>(s, out, tile, count, st);
}

}  // namespace dgs

using namespace dgs;

extern "C" size_t dgs_orthogonalise_workspace(const dgs_orthogonalise_args *args)
{
    if (!args || ortho_refused(*args) != DGS_OK || args->count == 0) return 0;
    return (size_t)ortho_plan(*args).bytes;
}

extern "C" int dgs_orthogonalise(const dgs_orthogonalise_args *args, void *hip_stream)
{
    if (!args) return DGS_EINVAL;
    const dgs_orthogonalise_args &p = *args;
    const int rc = ortho_refused(p);
    if (rc != DGS_OK) return rc;
    if (p.count == 0) return DGS_OK;
    if (!p.in || !p.out) return DGS_EINVAL;
    for (uint32_t i = 0; i < p.count; ++i)
        if (!matrix_ok(p.in[i].data, p.in[i].stride, p.cols, p.type) || !matrix_ok(p.out[i].data, p.out[i].stride, p.cols, p.out_type))
            return DGS_EINVAL;
    if (!p.workspace || !aligned_to(p.workspace, 16)) return DGS_EINVAL;
    const OrthoPlan o = ortho_plan(p);
    if (p.workspace_bytes < o.bytes) return DGS_ENOMEM;
    const hipStream_t st = (hipStream_t)hip_stream;
    const Coefficients by = {p.a, p.b, p.c};
    const uint32_t kind = o.two ? BOTH_IN_TWO : ONE_PAIR;
    for (uint32_t first = 0; first < p.count; first += o.at_once) {
        const uint32_t count = p.count - first < o.at_once ? p.count - first : o.at_once;
        Matrices in = {}, out = {};
        for (uint32_t i = 0; i < count; ++i) {
            in.data[i] = p.in[first + i].data;
            in.stride[i] = p.in[first + i].stride;
            out.data[i] = p.out[first + i].data;
            out.stride[i] = p.out[first + i].stride;
        }
        if (o.cols <= SMALL_SIDE) {
            const SmallArgs a = {p.rows, p.cols, (uint32_t)o.turned, (uint32_t)p.type, (uint32_t)p.out_type, p.steps, kind, (uint32_t)(p.accumulate != 0),
                                 by, p.eps, p.scale};
            if (o.cols <= 64) hipLaunchKernelGGL(k_ortho_small<64>, dim3(count), dim3(Small<64>::THREADS), 0, st, a, in, out);
            else hipLaunchKernelGGL(k_ortho_small<128>, dim3(count), dim3(Small<128>::THREADS), 0, st, a, in, out);
            continue;
        }
        if (p.type == DGS_F32) load_matrices<float>(in, p, o, count, st);
        else if (p.type == DGS_F16) load_matrices<f16>(in, p, o, count, st);
        else load_matrices<bf16>(in, p, o, count, st);
        float us = 0.0f;
        const int step_tile = product_tile([&](uint32_t high, uint32_t wide) { return (uint64_t)tiles_of(o.rows, high) * tiles_of(o.cols, wide) * count; },
                                           tiles_of(o.rows, PRODUCT_STEP) * (o.two ? 3u : 1u), TILE_256, us);
        for (uint32_t step = 0; step < p.steps; ++step) {
            SquareArgs g = {};
            g.x = o.x[step & 1u];
            g.depth = o.cols;
            g.kind = kind;
            g.size = o.rows;
            g.count = count;
            g.out = o.gram;
            g.bound = o.bound[step & 1u];
            launch_square<false>(g, o.square, o.sums, st);
            g.x = o.gram;
            g.bound = nullptr;
            g.depth = o.rows;
            g.out = o.poly;
            g.gram = o.gram;
            g.diagonal = o.diagonal;
            g.by = by;
            launch_square<true>(g, o.poly_square, o.sums, st);
            StepArgs s = {};
            s.poly = o.poly;
            s.x = o.x[step & 1u];
            if (step + 1 < p.steps) s.next = o.x[(step + 1) & 1u];
            s.diagonal = o.diagonal;
            s.rows = o.rows;
            s.cols = o.cols;
            s.kind = kind;
            s.bound = o.bound[step & 1u];
            s.next_bound = o.bound[(step + 1) & 1u];
            s.by = by;
            s.add = p.accumulate != 0;
            s.scale = p.scale;
            s.m_tiles = tiles_of(o.rows, tile_high(step_tile));
            s.n_tiles = tiles_of(o.cols, tile_high(step_tile));
            if (step + 1 < p.steps) launch_step<void, false>(s, out, step_tile, count, st);
            else if (p.out_type == DGS_F32) launch_last<float>(s, out, o.turned, step_tile, count, st);
            else if (p.out_type == DGS_F16) launch_last<f16>(s, out, o.turned, step_tile, count, st);
            else launch_last<bf16>(s, out, o.turned, step_tile, count, st);
        }
    }
    return launched();
}
