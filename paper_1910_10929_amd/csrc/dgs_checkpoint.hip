// Checkpoints of a matrix in 8 bits: encode and decode.
#include "dgs_rows.h"

namespace dgs {

constexpr uint32_t CKPT_THREADS = 256;

// One lane per eight columns of a row, four lanes to a run: its maximum is theirs, exchanged among them.  A row's lanes are
// padded to quads, so that a run never shares a quad with the next row's.  Bound by memory, 1 + 1/32 bytes a value beside the
// matrix: 65536 x 2304 of bfloat16, 458 MB, in 87 us (5.3 TB/s; a large copy reaches 5.0 to 5.4 on this card).
template <class T>
__global__ __launch_bounds__(CKPT_THREADS) void k_checkpoint_encode(const T *x, uint64_t x_stride, int8_t *codes, uint8_t *exps,
                                                                    uint64_t codes_stride, uint64_t exps_stride, uint32_t rows,
                                                                    uint32_t cols, uint32_t row_lanes)
{
    const uint64_t at = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x;
    const uint64_t row = at / row_lanes;
    const uint32_t c = (uint32_t)(at - row * row_lanes) * 8u;
    const uint32_t n = row < rows ? live8(c, cols) : 0u;
    float v[8];
    unpack8(load8(x + (n ? row * x_stride + c : 0u), n), v);
    save8(codes + row * codes_stride, exps + row * exps_stride, c, n, v);
}

// Lanes as above.  Bound by memory: the same matrix back, 458 MB in 73 us (6.3 TB/s, part of it from cache).
template <class T>
__global__ __launch_bounds__(CKPT_THREADS) void k_checkpoint_decode(const int8_t *codes, const uint8_t *exps, T *out,
                                                                    const float *scale, const float *shift, uint64_t codes_stride,
                                                                    uint64_t exps_stride, uint64_t out_stride, uint32_t rows,
                                                                    uint32_t cols, uint32_t row_lanes)
{
    const uint64_t at = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x;
    const uint64_t row = at / row_lanes;
    const uint32_t c = (uint32_t)(at - row * row_lanes) * 8u;
    const uint32_t n = row < rows ? live8(c, cols) : 0u;
    if (n == 0) return;
    uint32_t q[2];
    load_codes(codes + row * codes_stride + c, n, q);
    float v[8], w[8];
    decode8(q, run_scale(exps[row * exps_stride + c / DGS_CHECKPOINT_RUN]), v);
    if (scale) {
        load8_f32(scale + c, n, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    if (shift) {
        load8_f32(shift + c, n, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
    if (sizeof(T) == 2 && !scale && !shift) {
        // a code's value may lie above the largest half, by less than half a step, where the value itself did not
        if constexpr (__is_same(T, f16)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = v[i] != v[i] ? v[i] : min(max(v[i], -65504.0f), 65504.0f);
        }
    }
    store8(out + row * out_stride, c, n, v);
}

struct Shape {
    uint32_t row_lanes;
    uint64_t blocks;
};
static Shape shape_of(uint32_t rows, uint32_t cols)
{
    Shape s;
    s.row_lanes = (cols + DGS_CHECKPOINT_RUN - 1) / DGS_CHECKPOINT_RUN * (DGS_CHECKPOINT_RUN / 8);
    s.blocks = ((uint64_t)rows * s.row_lanes + CKPT_THREADS - 1) / CKPT_THREADS;
    return s;
}

template <class T>
static void encode(uint32_t rows, uint32_t cols, const void *x, uint64_t x_stride, const dgs_codes &to, const Shape &s, void *st)
{
    hipLaunchKernelGGL(k_checkpoint_encode<T>, dim3((uint32_t)s.blocks), dim3(CKPT_THREADS), 0, (hipStream_t)st, (const T *)x, x_stride,
                       to.codes, to.exps, to.codes_stride, to.exps_stride, rows, cols, s.row_lanes);
}
template <class T>
static void decode(uint32_t rows, uint32_t cols, const dgs_codes &from, const float *scale, const float *shift, void *out,
                   uint64_t out_stride, const Shape &s, void *st)
{
    hipLaunchKernelGGL(k_checkpoint_decode<T>, dim3((uint32_t)s.blocks), dim3(CKPT_THREADS), 0, (hipStream_t)st, from.codes, from.exps,
                       (T *)out, scale, shift, from.codes_stride, from.exps_stride, out_stride, rows, cols, s.row_lanes);
}

}  // namespace dgs

using namespace dgs;

extern "C" int dgs_checkpoint_encode(uint32_t rows, uint32_t cols, int type, const void *x, uint64_t x_stride,
                                     const dgs_codes *to, void *hip_stream)
{
    if (!to || cols == 0 || !is_type(type)) return DGS_EINVAL;
    if (rows == 0) return DGS_OK;
    if (!matrix_ok(x, x_stride, cols, type) || !codes_ok(*to, cols)) return DGS_EINVAL;
    const Shape s = shape_of(rows, cols);
    if (cols >= (1u << 29) || s.blocks > 0xFFFFFFull) return DGS_ENOTSUP;
    if (type == DGS_F32) encode<float>(rows, cols, x, x_stride, *to, s, hip_stream);
    else if (type == DGS_F16) encode<f16>(rows, cols, x, x_stride, *to, s, hip_stream);
    else encode<bf16>(rows, cols, x, x_stride, *to, s, hip_stream);
    return launched();
}

extern "C" int dgs_checkpoint_decode(uint32_t rows, uint32_t cols, const dgs_codes *from, const float *scale,
                                     const float *shift, int type, void *out, uint64_t out_stride, void *hip_stream)
{
    if (!from || cols == 0 || !is_type(type) || !aligned_to(scale, 4) || !aligned_to(shift, 4)) return DGS_EINVAL;
    if (rows == 0) return DGS_OK;
    if (!matrix_ok(out, out_stride, cols, type) || !codes_ok(*from, cols)) return DGS_EINVAL;
    const Shape s = shape_of(rows, cols);
    if (cols >= (1u << 29) || s.blocks > 0xFFFFFFull) return DGS_ENOTSUP;
    if (type == DGS_F32) decode<float>(rows, cols, *from, scale, shift, out, out_stride, s, hip_stream);
    else if (type == DGS_F16) decode<f16>(rows, cols, *from, scale, shift, out, out_stride, s, hip_stream);
    else decode<bf16>(rows, cols, *from, scale, shift, out, out_stride, s, hip_stream);
    return launched();
}
