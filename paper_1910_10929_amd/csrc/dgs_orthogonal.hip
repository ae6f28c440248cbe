// Updates orthogonalised by Newton-Schulz products: X = G / (|G| + eps), then `steps` times with A = X X^T
//
//     X = a X + (b A + c A^2) X
//
// which leaves G's singular vectors and takes its singular values towards 1 (X^T in place of X where rows outnumber columns, so
// that A is the smaller square).  Three launches a step: the two symmetric products, of which tiles on and below the diagonal
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
constexpr uint32_t NORM_PARTS = 64;

struct Matrices {
    const void *data[ORTHO_AT_ONCE];
    uint64_t stride[ORTHO_AT_ONCE];
};
struct Halves {
    uint16_t *hi, *lo;
    uint64_t stride, size;      // from row to row, and of a matrix
};

// An update whose norm is far below eps starts with an X far below 1, which grows by `a` a step at most.  X is then held times
// 2^lift besides, so that what half's smallest numbers cut off stays as far below it as ever.  growth: log2(a^step).
__device__ __forceinline__ int lift_of(float log2_norm, float growth)
{
    const float down = -(log2_norm + growth);
    return down >= 1.0f ? (int)min(down, 120.0f) : 0;      // (a NaN: 0)
}
__device__ __forceinline__ float times_power(float v, int e)
{
#ifdef DGS_HOST_EMULATION
    return ldexpf(v, e);
#else
    return __builtin_amdgcn_ldexpf(v, e);
#endif
}
__device__ __forceinline__ float value_of(uint16_t bits)
{
    f16 h;
    __builtin_memcpy(&h, &bits, 2);
    return (float)h;
}
__device__ __forceinline__ uint16_t half_bits(f16 h)
{
    uint16_t b;
    __builtin_memcpy(&b, &h, 2);
    return b;
}

// Sums of squares, NORM_PARTS a matrix.
template <class T>
__global__ __launch_bounds__(256) void k_ortho_norm(Matrices in, uint32_t rows, uint32_t cols, double *parts)
{
    __shared__ double sums[256];
    const uint32_t which = blockIdx.y;
    const T *const m = (const T *)in.data[which];
    const uint64_t stride = in.stride[which], pieces = (cols + 7) / 8, end = pieces * rows;
    double s = 0.0;
    for (uint64_t at = blockIdx.x * 256 + threadIdx.x; at < end; at += NORM_PARTS * 256) {
        const uint64_t row = at / pieces;
        const uint32_t c = (uint32_t)(at - row * pieces) * 8;
        float v[8];
        unpack8(load8(m + row * stride + c, live8(c, cols)), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += (double)v[i] * (double)v[i];
    }
    sums[threadIdx.x] = s;
    __syncthreads();
    for (uint32_t by = 128; by; by >>= 1) {
        if (threadIdx.x < by) sums[threadIdx.x] += sums[threadIdx.x + by];
        __syncthreads();
    }
    if (threadIdx.x == 0) parts[which * NORM_PARTS + blockIdx.x] = sums[0];
}

// X from G, 64 x 64 of it to a workgroup, turned where that makes it wide.  Columns up to a multiple of eight are zeros.
template <class T>
__global__ __launch_bounds__(256) void k_ortho_load(Matrices in, uint32_t rows, uint32_t cols, uint32_t turned, const double *parts,
                                                    float eps, Halves x, float *log2_norm)
{
    __shared__ double norm[NORM_PARTS];
    __shared__ float tile[64][65];
    const uint32_t which = blockIdx.y, across = (cols + 63) / 64;
    if (threadIdx.x < NORM_PARTS) norm[threadIdx.x] = parts[which * NORM_PARTS + threadIdx.x];
    __syncthreads();
    double sum = 0.0;
    for (uint32_t i = 0; i < NORM_PARTS; ++i) sum += norm[i];
    const double length = sqrt(sum), whole = length + (double)eps;
    const float log2_of = sum > 0.0 ? (float)(log2(length) - log2(whole)) : 0.0f;
    const double by = ldexp((double)HELD, lift_of(log2_of, 0.0f)) / whole;
    if (blockIdx.x == 0 && threadIdx.x == 0) log2_norm[which] = log2_of;
    const T *const m = (const T *)in.data[which];
    const uint64_t stride = in.stride[which];
    const uint32_t r0 = blockIdx.x / across * 64, c0 = blockIdx.x % across * 64;      // of G
    const uint32_t c = c0 + (threadIdx.x & 63u);
    for (uint32_t i = threadIdx.x >> 6; i < 64; i += 4) {
        const uint32_t r = r0 + i;
        tile[i][threadIdx.x & 63u] = r < rows && c < cols ? (float)((double)to_float(m[r * stride + c]) * by) : 0.0f;
    }
    __syncthreads();
    const uint32_t x_rows = turned ? cols : rows;
    const uint32_t first_row = turned ? c0 : r0, first_col = turned ? r0 : c0;
    for (uint32_t at = threadIdx.x; at < 64 * 16; at += 256) {
        const uint32_t i = at >> 4, q = (at & 15u) * 4;
        if (first_row + i >= x_rows || first_col + q >= x.stride) continue;
        f16 hi[4], lo[4];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) halves_of(turned ? tile[q + k][i] : tile[i][q + k], hi[k], lo[k]);
        const uint64_t to = which * x.size + (first_row + i) * x.stride + first_col + q;
        u32x2 o;
        o[0] = bits_of(hi[0], hi[1]);
        o[1] = bits_of(hi[2], hi[3]);
        *(u32x2 *)(x.hi + to) = o;
        o[0] = bits_of(lo[0], lo[1]);
        o[1] = bits_of(lo[2], lo[3]);
        *(u32x2 *)(x.lo + to) = o;
    }
}

struct SquareArgs {
    Halves x;                // both operands: rows of it by rows of it
    uint32_t depth, kind;
    uint32_t size, tiles;    // of the result, and tiles along a side
    const float *log2_norm;  // of each X at the start; absent: nothing was lifted
    float growth;            // of X since
    Halves out;              // lo: absent where products take the first halves
    // the polynomial: b A + c A^2, and its diagonal
    Halves gram;
    float *diagonal;         // size a matrix
    float a, b, c;
};

// The symmetric product of X with itself (POLY: of A with itself, from which the polynomial is made).
template <uint32_t M, uint32_t WAVES_M, uint32_t WAVES_N, bool POLY>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64, 2) void k_ortho_square(SquareArgs a)
{
    typedef Product<f16, M, M, WAVES_M, WAVES_N, false, false> P;
    __shared__ __attribute__((aligned(16))) typename P::Lds lds;
    // tiles on and below the diagonal, row by row
    const uint32_t count = a.tiles * (a.tiles + 1) / 2;
    const uint32_t all = tile_of_block(blockIdx.x, gridDim.x), which = all / count, at = all - which * count;
    uint32_t tile_m = 0, passed = 0;
    while (passed + tile_m + 1 <= at) passed += ++tile_m;
    const uint32_t tile_n = at - passed;
    const Side side = {{a.x.hi + which * a.x.size, a.x.lo ? a.x.lo + which * a.x.size : nullptr}, a.x.stride, a.size};
    typename P::Sums s;
    P::run(lds, side, side, tile_m * M, tile_n * M, 0, a.depth, a.kind, s);
    const uint32_t half = lane_id() >> 5;
    const uint64_t base = which * a.out.size;
    const int power = -12 - (a.log2_norm ? 2 * lift_of(a.log2_norm[which], a.growth) : 0);
#pragma unroll
    for (uint32_t j = 0; j < P::J; ++j) {
        const uint32_t n = tile_n * M + P::wave_n() + 32 * j + (lane_id() & 31u);
        if (n >= a.out.stride) continue;
#pragma unroll
        for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
            for (uint32_t g = 0; g < 4; ++g) {
                const uint32_t m = tile_m * M + P::wave_m() + 32 * i + 8 * g + 4 * half;
                if (m >= a.out.stride) continue;
                float v[4];
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) v[q] = times_power(s[i][j][4 * g + q], power);
                if constexpr (POLY) {
                    u32x2 hi = {0, 0}, lo = {0, 0};
                    const uint64_t from = which * a.gram.size + n * a.gram.stride + m;
                    if (n < a.size) {
                        hi = *(const u32x2 *)(a.gram.hi + from);
                        if (a.gram.lo) lo = *(const u32x2 *)(a.gram.lo + from);
                    }
#pragma unroll
                    for (uint32_t q = 0; q < 4; ++q) {
                        const float gram = value_of((uint16_t)(hi[q >> 1] >> (16 * (q & 1)))) + value_of((uint16_t)(lo[q >> 1] >> (16 * (q & 1))));
                        v[q] = a.b * gram + a.c * v[q];
                        if (m + q == n) {
                            if (n < a.size) a.diagonal[which * a.size + n] = a.a + v[q] * LEFT;
                            v[q] = 0.0f;
                        }
                    }
                }
                f16 hi[4], lo[4];
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) halves_of(v[q], hi[q], lo[q]);
                if (n < a.size) {
                    u32x2 o;
                    const uint64_t to = base + n * a.out.stride + m;
                    o[0] = bits_of(hi[0], hi[1]);
                    o[1] = bits_of(hi[2], hi[3]);
                    *(u32x2 *)(a.out.hi + to) = o;
                    if (a.out.lo) {
                        o[0] = bits_of(lo[0], lo[1]);
                        o[1] = bits_of(lo[2], lo[3]);
                        *(u32x2 *)(a.out.lo + to) = o;
                    }
                }
                if (tile_m == tile_n) continue;
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) {
                    if (m + q >= a.size) continue;
                    const uint64_t to = base + (m + q) * a.out.stride + n;
                    a.out.hi[to] = half_bits(hi[q]);
                    if (a.out.lo) a.out.lo[to] = half_bits(lo[q]);
                }
            }
    }
}

struct StepArgs {
    Halves poly, x, next;      // next.hi: absent in the last step
    const float *diagonal;
    uint32_t rows, cols, kind;
    uint32_t m_tiles, n_tiles;
    const float *log2_norm;
    float growth, next_growth;
    // the last step
    uint32_t turned, add;
    int32_t out_type;
    float scale;
    Matrices out;
};

template <class T> __device__ __forceinline__ void put(T *p, float v, uint32_t add)
{
    *p = from_float<T>(add ? to_float(*p) + v : v);
}

// X of the next step: its rows times the polynomial's diagonal, plus the product of the rest with it.
template <uint32_t M, uint32_t N, uint32_t WAVES_M, uint32_t WAVES_N>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64, 2) void k_ortho_step(StepArgs a)
{
    typedef Product<f16, M, N, WAVES_M, WAVES_N, false, true> P;
    __shared__ __attribute__((aligned(16))) typename P::Lds lds;
    const uint32_t count = a.m_tiles * a.n_tiles;
    const uint32_t all = tile_of_block(blockIdx.x, gridDim.x), which = all / count, at = all - which * count;
    const uint32_t tile_m = at / a.n_tiles, tile_n = at - tile_m * a.n_tiles;
    const uint16_t *const x_hi = a.x.hi + which * a.x.size, *const x_lo = a.x.lo + which * a.x.size;
    const Side left = {{a.poly.hi + which * a.poly.size, a.poly.lo ? a.poly.lo + which * a.poly.size : nullptr}, a.poly.stride, a.rows};
    const Side right = {{x_hi, x_lo}, a.x.stride, a.cols};
    typename P::Sums s;
    P::run(lds, left, right, tile_m * M, tile_n * N, 0, a.rows, a.kind, s);
    // from how this X is held to how the next one is, or to the result
    const int lift = lift_of(a.log2_norm[which], a.growth);
    const int power = a.next.hi ? lift_of(a.log2_norm[which], a.next_growth) - lift : -12 - lift;
#pragma unroll
    for (uint32_t i = 0; i < P::I; ++i)
#pragma unroll
        for (uint32_t r = 0; r < 16; ++r) {
            const uint32_t m = tile_m * M + P::wave_m() + 32 * i + square_row(r);
            if (m >= a.rows) continue;
            const float d = a.diagonal[which * a.rows + m];
#pragma unroll
            for (uint32_t j = 0; j < P::J; ++j) {
                const uint32_t n = tile_n * N + P::wave_n() + 32 * j + (lane_id() & 31u);
                if (n >= a.x.stride) continue;
                const uint64_t here = m * a.x.stride + n;
                const float x = value_of(x_hi[here]) + value_of(x_lo[here]);
                const float v = times_power(__builtin_fmaf(d, x, s[i][j][r] * LEFT), power);
                if (a.next.hi) {
                    f16 hi, lo;
                    halves_of(v, hi, lo);
                    a.next.hi[which * a.next.size + here] = half_bits(hi);
                    a.next.lo[which * a.next.size + here] = half_bits(lo);
                } else if (n < a.cols) {
                    const uint64_t stride = a.out.stride[which], to = a.turned ? n * stride + m : m * stride + n;
                    const float w = v * a.scale;
                    void *const out = (void *)a.out.data[which];
                    if (a.out_type == DGS_F32) put((float *)out + to, w, a.add);
                    else if (a.out_type == DGS_F16) put((f16 *)out + to, w, a.add);
                    else put((bf16 *)out + to, w, a.add);
                }
            }
        }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

struct OrthoPlan {
    uint32_t rows, cols, at_once;      // of X, and matrices of a launch
    bool turned, two;
    Halves x[2], gram, poly;
    double *norm;
    float *diagonal, *log2_norm;
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
    o.log2_norm = (float *)s.take(4ull * o.at_once);
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
    hipLaunchKernelGGL(k_ortho_norm<T>, dim3(NORM_PARTS, count), dim3(256), 0, st, in, p.rows, p.cols, o.norm);
    hipLaunchKernelGGL(k_ortho_load<T>, dim3((p.cols + 63) / 64 * ((p.rows + 63) / 64), count), dim3(256), 0, st, in, p.rows, p.cols,
                       (uint32_t)o.turned, (const double *)o.norm, p.eps, o.x[0], o.log2_norm);
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
    for (uint32_t first = 0; first < p.count; first += o.at_once) {
        const uint32_t count = p.count - first < o.at_once ? p.count - first : o.at_once;
        Matrices in = {}, out = {};
        for (uint32_t i = 0; i < count; ++i) {
            in.data[i] = p.in[first + i].data;
            in.stride[i] = p.in[first + i].stride;
            out.data[i] = p.out[first + i].data;
            out.stride[i] = p.out[first + i].stride;
        }
        if (p.type == DGS_F32) load_matrices<float>(in, p, o, count, st);
        else if (p.type == DGS_F16) load_matrices<f16>(in, p, o, count, st);
        else load_matrices<bf16>(in, p, o, count, st);
        const uint32_t kind = o.two ? BOTH_IN_TWO : ONE_PAIR;
        auto tiles = [](uint32_t n, uint32_t size) { return (n - 1) / size + 1; };
        const uint32_t t256 = tiles(o.rows, 256);
        bool large_square = (uint64_t)t256 * (t256 + 1) / 2 * count >= 192;
        bool large_step = (uint64_t)t256 * tiles(o.cols, 256) * count >= 192;
#ifdef DGS_ORTHO_LARGE      // (a CPU build that is to reach one kind on small matrices)
        large_square = large_step = DGS_ORTHO_LARGE;
#endif
        const float grows = p.a != 0.0f ? log2f(fabsf(p.a)) : 0.0f;
        const uint32_t side = tiles(o.rows, large_square ? 256 : 128);
        for (uint32_t step = 0; step < p.steps; ++step) {
            SquareArgs g = {};
            g.x = o.x[step & 1u];
            g.depth = o.cols;
            g.kind = kind;
            g.size = o.rows;
            g.tiles = side;
            g.out = o.gram;
            g.log2_norm = o.log2_norm;
            g.growth = (float)step * grows;
            const dim3 grid(side * (side + 1) / 2 * count);
            if (large_square) hipLaunchKernelGGL((k_ortho_square<256, 2, 4, false>), grid, dim3(512), 0, st, g);
            else hipLaunchKernelGGL((k_ortho_square<128, 2, 2, false>), grid, dim3(256), 0, st, g);
            g.x = o.gram;
            g.log2_norm = nullptr;
            g.depth = o.rows;
            g.out = o.poly;
            g.gram = o.gram;
            g.diagonal = o.diagonal;
            g.a = p.a;
            g.b = p.b;
            g.c = p.c;
            if (large_square) hipLaunchKernelGGL((k_ortho_square<256, 2, 4, true>), grid, dim3(512), 0, st, g);
            else hipLaunchKernelGGL((k_ortho_square<128, 2, 2, true>), grid, dim3(256), 0, st, g);
            StepArgs s = {};
            s.poly = o.poly;
            s.x = o.x[step & 1u];
            if (step + 1 < p.steps) s.next = o.x[(step + 1) & 1u];
            s.diagonal = o.diagonal;
            s.rows = o.rows;
            s.cols = o.cols;
            s.kind = kind;
            s.log2_norm = o.log2_norm;
            s.growth = (float)step * grows;
            s.next_growth = s.growth + grows;
            s.turned = o.turned;
            s.add = p.accumulate != 0;
            s.out_type = p.out_type;
            s.scale = p.scale;
            s.out = out;
            const uint32_t size = large_step ? 256 : 128;
            s.m_tiles = tiles(o.rows, size);
            s.n_tiles = tiles(o.cols, size);
            const dim3 all(s.m_tiles * s.n_tiles * count);
            if (large_step) hipLaunchKernelGGL((k_ortho_step<256, 256, 2, 4>), all, dim3(512), 0, st, s);
            else hipLaunchKernelGGL((k_ortho_step<128, 128, 2, 2>), all, dim3(256), 0, st, s);
        }
    }
    return launched();
}
