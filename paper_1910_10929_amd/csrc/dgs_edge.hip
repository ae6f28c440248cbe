// The edge between two blocks: norm of the branch, gate, residual sum and norm of the stream in one pass over the rows, and
// its gradients in another.
//
// A row belongs to a team of wavefronts that holds all of it in registers, eight consecutive columns in a lane, so that the
// statistics are taken of what is there (mean first, then the squares of what is left) and every matrix is read and written
// once.  The next row's loads are issued piece by piece while a row is worked on; no load stands in a branch, so that a wait
// is for what is due and not for all that is under way.  Parameters stay in registers from row to row (backward: in LDS).
//
// Bound by memory where there are rows enough.  Calls among others, two launches where there are partial sums: forward 8192 x
// 768, fp32 stream, bfloat16 branch, checkpoints, 88.6 MB in 18.0 us (4.9 TB/s), 16384 x 4096 of bfloat16 with a gate a row, 809 MB
// in 154 us (5.3); backward 8192 x 768 25.5 us (88.6 MB, 3.5 TB/s: 16 wavefronts of one workgroup to a compute unit, four rounds of
// eight rows each), 16384 x 4096, 675 MB in 141 us (4.8).  Kernels by themselves, from a chip that has come to rest: 19.2, 147,
// 24.8 + 4.0 and 152 + 5.2 us.  A single row of 768: 3.6 us forward, all of it latency.
#include "dgs_rows.h"

namespace dgs {

struct EdgeLayer {
    const float *post_weight, *post_bias, *pre_weight, *pre_bias;
    uint32_t cols;
    int32_t post, pre;
    float post_eps, pre_eps, skip, branch, inv_cols;
};

struct ForwardArgs {
    EdgeLayer l;
    const void *x, *f, *gate;
    void *x_out, *u;
    int8_t *post_codes, *pre_codes;
    uint8_t *post_exps, *pre_exps;
    float *stats;
    uint32_t x_stride, f_stride, gate_stride, x_out_stride, u_stride;
    uint32_t post_codes_stride, post_exps_stride, pre_codes_stride, pre_exps_stride;
    uint32_t rows, rows_per_gate, gate_f32, branch, gated;      // branch, gated: there is one
};

// 1 / sqrt(v), v > 0 (1 ulp)
__device__ __forceinline__ float rsqrt_of(float v)
{
#ifdef DGS_HOST_EMULATION
    return 1.0f / sqrtf(v);
#else
    return __builtin_amdgcn_rsqf(v);
#endif
}

// A gate's eight values: fp32, or of the branch's type (which is then loaded twice, so that the number of loads does not
// depend on the type).
struct GateRaw { u32x4_any lo, hi; };
template <bool TINY, class TF>
__device__ __forceinline__ GateRaw load_gate(const void *gate, uint64_t row_at, uint32_t at, uint32_t cols, bool f32)
{
    GateRaw g;
    if constexpr (TINY) {
        if (f32) {
            const Raw8<float> r = load_at<true>((const float *)gate + row_at, at, cols);
            __builtin_memcpy(&g, &r, sizeof(r));
        } else {
            const Raw8<TF> r = load_at<true>((const TF *)gate + row_at, at, cols);
            __builtin_memcpy(&g, &r, sizeof(r));
        }
    } else {
        const uint32_t bytes = f32 ? 4u : (uint32_t)sizeof(TF);
        const char *const row = (const char *)gate + row_at * bytes;
        const uint32_t o = opaque(at * bytes);
        g.lo = *(const u32x4_any *)(row + o);
        g.hi = *(const u32x4_any *)(row + (bytes == 4u ? 16u : 0u) + o);
    }
    return g;
}
template <bool TINY, class TF>
__device__ __forceinline__ void unpack_gate(const GateRaw &g, bool f32, bool ragged, const Place8 &p, float (&v)[8])
{
    if (f32) {
        Raw8<float> r;
        __builtin_memcpy(&r, &g, sizeof(r));
        if (ragged) in_place<TINY>(r, p);
        unpack8(r, v);
    } else {
        Raw8<TF> r;
        __builtin_memcpy(&r, &g, sizeof(r));
        if (ragged) in_place<TINY>(r, p);
        unpack8(r, v);
    }
}

// Teams of a forward workgroup where they are single wavefronts (otherwise it is one team); wavefronts of a backward workgroup,
// whatever its teams: fewer workgroups leave fewer partial sums (with 8, two workgroups to a compute unit, 16384 x 4096 takes
// 151 us in place of 141, 8192 x 768 27.3 in place of 25.6, 20000 x 2100 126 in place of 121, 777 x 1001 of fp32 19.6 in place of 19.4).
constexpr uint32_t FORWARD_TEAMS = 4;
constexpr int backward_wavefronts(int waves) { return waves % 3 == 0 ? 12 : 16; }
constexpr uint32_t BACKWARD_BLOCKS = 256;

template <int WAVES, int CHUNKS> struct Team {
    static constexpr uint32_t LANES = WAVES * 64;
    // first column of this lane's k-th eight
    static __device__ __forceinline__ uint32_t col(int k) { return ((uint32_t)k * LANES + threadIdx.x % LANES) * 8u; }
};

// Whether a team's row ends before this wavefront's first column (CHUNKS = 1).
template <int WAVES> __device__ __forceinline__ bool idle_wave(uint32_t cols)
{
    return uniform((threadIdx.x / 64 % WAVES) * 512u) >= cols;
}

// v - by, and 0 behind the row's end in the lane that holds it (where the row's length is no multiple of eight).
template <int CHUNKS>
__device__ __forceinline__ void subtract(float (&v)[CHUNKS][8], const Place8 (&p)[CHUNKS], bool ragged, float by)
{
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] -= by;
        if (ragged) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = (uint32_t)i < p[k].n ? v[k][i] : 0.0f;
        }
    }
}

// Statistics of a row and its normalised values, in place.
template <int WAVES, int ALL, int CHUNKS>
__device__ __forceinline__ void normalise(float (&v)[CHUNKS][8], const Place8 (&p)[CHUNKS], bool ragged, int kind, float eps,
                                          float inv_cols, TeamLds<ALL> &lds, uint32_t &turn, float &mean, float &rstd)
{
    mean = rstd = 0.0f;
    if (kind == DGS_NORM_NONE) return;
    float s[1];
    if (kind == DGS_NORM_LAYER) {
        s[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            float of_lane = v[k][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) of_lane += v[k][i];
            s[0] += p[k].n ? of_lane : 0.0f;
        }
        team_sum<WAVES, ALL, 1>(s, lds, turn);
        mean = s[0] * inv_cols;
        subtract<CHUNKS>(v, p, ragged, mean);
    }
    s[0] = 0.0f;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        float of_lane = v[k][0] * v[k][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) of_lane = __builtin_fmaf(v[k][i], v[k][i], of_lane);
        s[0] += p[k].n ? of_lane : 0.0f;
    }
    team_sum<WAVES, ALL, 1>(s, lds, turn);
    rstd = rsqrt_of(__builtin_fmaf(s[0], inv_cols, eps));
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] *= rstd;
}

// The forward pass, a row to a team.
template <class TX, class TF, int WAVES, int CHUNKS, bool TINY>
__global__ __launch_bounds__(WAVES == 1 ? FORWARD_TEAMS * 64 : WAVES * 64) void k_edge_forward(ForwardArgs a)
{
    constexpr uint32_t TEAMS = WAVES == 1 ? FORWARD_TEAMS : 1;
    constexpr int ALL = TEAMS * WAVES;
    __shared__ TeamLds<ALL> lds;
    uint32_t turn = 0;
    const uint32_t team = uniform(blockIdx.x * TEAMS + threadIdx.x / (WAVES * 64));
    const uint32_t teams = gridDim.x * TEAMS;
    const EdgeLayer &l = a.l;
    const bool ragged = TINY || (l.cols & 7u) != 0;
    Place8 p[CHUNKS];
    float wp[CHUNKS][8], bp[CHUNKS][8], wn[CHUNKS][8], bn[CHUNKS][8];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        p[k] = place8<TINY>(Team<WAVES, CHUNKS>::col(k), l.cols);
        if (l.post_weight) load8_f32(l.post_weight + p[k].c, p[k].n, wp[k]);
        if (l.post_bias) load8_f32(l.post_bias + p[k].c, p[k].n, bp[k]);
        if (l.pre_weight) load8_f32(l.pre_weight + p[k].c, p[k].n, wn[k]);
        if (l.pre_bias) load8_f32(l.pre_bias + p[k].c, p[k].n, bn[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!l.post_weight) wp[k][i] = 1.0f;
            if (!l.post_bias) bp[k][i] = 0.0f;
            if (!l.pre_weight) wn[k][i] = 1.0f;
            if (!l.pre_bias) bn[k][i] = 0.0f;
        }
    }
    uint32_t row = team;
    if (row >= a.rows) return;      // (of a workgroup that is one team, all of it)
    if (WAVES > 1 && idle_wave<WAVES>(l.cols)) {      // (nothing but the other wavefronts' sums)
        const uint32_t sums = (a.branch ? (uint32_t)l.post : 0u) + (uint32_t)l.pre;      // as `normalise` takes: RMS 1, layer norm 2
        for (; row < a.rows; row += teams)
            for (uint32_t i = 0; i < sums; ++i) {
                float none[1] = {0.0f};
                team_sum<WAVES, ALL, 1>(none, lds, turn);
            }
        return;
    }
    // What is loaded of a row (f and the gate, if there are none, of x in their place).  Each piece of the next row is asked for
    // as soon as this row's has been unpacked, so that it has a whole round to arrive and takes no registers of its own.  (With 16
    // columns a lane there are none for it: each piece is asked for when it is due.)
    constexpr bool AHEAD = CHUNKS == 1;
    Raw8<TX> raw_x[CHUNKS];
    Raw8<TF> raw_f[CHUNKS];
    GateRaw raw_g[CHUNKS];
    auto fetch_x = [&](uint32_t r) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) raw_x[k] = load_at<TINY>((const TX *)a.x + (uint64_t)r * a.x_stride, p[k].at, l.cols);
    };
    auto fetch_f = [&](uint32_t r) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) raw_f[k] = load_at<TINY>((const TF *)a.f + (uint64_t)r * a.f_stride, p[k].at, l.cols);
    };
    auto fetch_g = [&](uint32_t r) {
        const uint64_t gate_at = (uint64_t)(r / a.rows_per_gate) * a.gate_stride;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) raw_g[k] = load_gate<TINY, TF>(a.gate, gate_at, p[k].at, l.cols, a.gate_f32);
    };
    if constexpr (AHEAD) {
        fetch_f(row);
        fetch_x(row);
        fetch_g(row);
    }
    for (; row < a.rows; row += teams) {
        const uint32_t next = row + teams < a.rows ? row + teams : row;
        float x[CHUNKS][8], f[CHUNKS][8];
        float post_mean = 0.0f, post_rstd = 0.0f, pre_mean, pre_rstd;
        if constexpr (!AHEAD) fetch_f(row);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            if (ragged) in_place<TINY>(raw_f[k], p[k]);
            unpack8(raw_f[k], f[k]);
        }
        if constexpr (AHEAD) fetch_f(next);
        else fetch_x(row);
        if (a.branch) normalise<WAVES, ALL, CHUNKS>(f, p, ragged, l.post, l.post_eps, l.inv_cols, lds, turn, post_mean, post_rstd);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            if (ragged) in_place<TINY>(raw_x[k], p[k]);
            unpack8(raw_x[k], x[k]);
        }
        if constexpr (AHEAD) fetch_x(next);
        else fetch_g(row);
        if (a.branch) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                if (a.post_codes)
                    save8(a.post_codes + (uint64_t)row * a.post_codes_stride, a.post_exps + (uint64_t)row * a.post_exps_stride, p[k].c, p[k].n, f[k]);
                float g[8];
                unpack_gate<TINY, TF>(raw_g[k], a.gate_f32, ragged, p[k], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float m = a.gated ? l.branch * g[i] : l.branch;
                    x[k][i] = __builtin_fmaf(m, __builtin_fmaf(f[k][i], wp[k][i], bp[k][i]), l.skip * x[k][i]);
                }
                store8((TX *)a.x_out + (uint64_t)row * a.x_out_stride, p[k].c, p[k].n, x[k]);
            }
            // (behind the row's end the gate may be anything: not the sum)
            if (ragged) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[k][i] = (uint32_t)i < p[k].n ? x[k][i] : 0.0f;
            }
        }
        if constexpr (AHEAD) fetch_g(next);
        normalise<WAVES, ALL, CHUNKS>(x, p, ragged, l.pre, l.pre_eps, l.inv_cols, lds, turn, pre_mean, pre_rstd);
        if (l.pre != DGS_NORM_NONE) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                if (a.pre_codes)
                    save8(a.pre_codes + (uint64_t)row * a.pre_codes_stride, a.pre_exps + (uint64_t)row * a.pre_exps_stride, p[k].c, p[k].n, x[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[k][i] = __builtin_fmaf(x[k][i], wn[k][i], bn[k][i]);
                store8((TF *)a.u + (uint64_t)row * a.u_stride, p[k].c, p[k].n, x[k]);
            }
        }
        if (a.stats && threadIdx.x % (WAVES * 64) == 0) {
            f32x4_any s;
            s.x = post_mean; s.y = post_rstd; s.z = pre_mean; s.w = pre_rstd;
            *(f32x4_any *)(a.stats + 4 * (uint64_t)row) = s;
        }
    }
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------

// How rows are dealt out to workgroups.  Every gate row's rows are cut into `parts` runs of `run` rows, one per workgroup,
// and the parts of its gradient are added up afterwards (one part: written at once); or, where there are many gate rows, a
// workgroup takes `whole` of them, each of which is one team's.
struct Cut {
    uint32_t blocks, whole, parts, run;
    uint32_t gates, rows_per_gate;
};

struct BackwardArgs {
    EdgeLayer l;
    Cut cut;
    const void *dx_out, *du, *gate, *f, *x_out;
    const int8_t *post_codes, *pre_codes;
    const uint8_t *post_exps, *pre_exps;
    const float *stats;
    void *dx, *df, *dgate;
    float *grad[4];         // post weight, post bias, pre weight, pre bias
    float *partial;         // 5 x blocks x cols (the fifth: the gate's)
    uint32_t dx_out_stride, du_stride, gate_stride, f_stride, x_out_stride, dx_stride, df_stride, dgate_stride;
    uint32_t post_codes_stride, post_exps_stride, pre_codes_stride, pre_exps_stride;
    uint32_t rows, gate_f32, accumulate, branch, gated, through_pre, arrives, coded;     // (branch .. arrives: there is such)
};

enum { ACC_POST_WEIGHT, ACC_POST_BIAS, ACC_PRE_WEIGHT, ACC_PRE_BIAS, ACC_GATE, ACCS };

// Normalised values as the forward pass left them: codes, or the values themselves.
template <class T, bool CODED> struct Kept;
template <class T> struct Kept<T, true> { uint32_t q[2], byte; };
template <class T> struct Kept<T, false> { Raw8<T> v; };

template <bool TINY, class T, bool CODED>
__device__ __forceinline__ void fetch_kept(Kept<T, CODED> &r, const int8_t *codes, const uint8_t *exps, uint32_t codes_stride,
                                           uint32_t exps_stride, const void *values, uint32_t stride, uint64_t row, const Place8 &p,
                                           uint32_t cols)
{
    if constexpr (CODED) {
        load_codes_at<TINY>(codes + row * codes_stride, p.at, cols, r.q);
        r.byte = (exps + row * exps_stride)[opaque(min(p.c, cols - 1u) / DGS_CHECKPOINT_RUN)];
    } else {
        r.v = load_at<TINY>((const T *)values + row * stride, p.at, cols);
    }
}
// The normalised row.
template <bool TINY, class T, bool CODED, int CHUNKS>
__device__ __forceinline__ void unpack_kept(Kept<T, CODED> (&r)[CHUNKS], int kind, float mean, float rstd, const Place8 (&p)[CHUNKS],
                                            bool ragged, float (&v)[CHUNKS][8])
{
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        if constexpr (CODED) {
            if (ragged) codes_in_place<TINY>(r[k].q, p[k]);
            decode8(r[k].q, run_scale(r[k].byte), v[k]);
        } else {
            if (ragged) in_place<TINY>(r[k].v, p[k]);
            unpack8(r[k].v, v[k]);
        }
    }
    if constexpr (!CODED) {
        if (kind == DGS_NORM_NONE) return;
        if (kind == DGS_NORM_LAYER) subtract<CHUNKS>(v, p, ragged, mean);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] *= rstd;
    }
}

// The gradient through a norm at its normalised output h, in place.
template <int WAVES, int ALL, int CHUNKS>
__device__ __forceinline__ void through_norm(float (&g)[CHUNKS][8], const float (&h)[CHUNKS][8], const Place8 (&p)[CHUNKS], bool ragged,
                                             int kind, float rstd, float inv_cols, TeamLds<ALL> &lds, uint32_t &turn)
{
    if (kind == DGS_NORM_NONE) return;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        float of_lane = g[k][0] * h[k][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) of_lane = __builtin_fmaf(g[k][i], h[k][i], of_lane);
        s[0] += p[k].n ? of_lane : 0.0f;
    }
    if (kind == DGS_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            float of_lane = g[k][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) of_lane += g[k][i];
            s[1] += p[k].n ? of_lane : 0.0f;
        }
        team_sum<WAVES, ALL, 2>(s, lds, turn);
        subtract<CHUNKS>(g, p, ragged, s[1] * inv_cols);
    } else {
        float one[1] = {s[0]};
        team_sum<WAVES, ALL, 1>(one, lds, turn);
        s[0] = one[0];
    }
    const float along = -s[0] * inv_cols;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) g[k][i] = __builtin_fmaf(along, h[k][i], g[k][i]) * rstd;
}

template <class T> __device__ __forceinline__ void store_grad8(T *row, uint32_t c, uint32_t n, float (&v)[8], bool add)
{
    if (add) {
        float o[8];
        unpack8(load8(row + c, n), o);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += o[i];
    }
    store8(row, c, n, v);
}

// A gate's gradient at one place.
template <class TF> __device__ __forceinline__ void store_gate(void *dgate, uint64_t at, bool f32, bool add, float v)
{
    if (f32) ((float *)dgate)[at] = add ? ((float *)dgate)[at] + v : v;
    else ((TF *)dgate)[at] = from_float<TF>(v);
}

// Eight parameters of the backward pass: staged in LDS, or where a row is too long for that (STAGED false) from memory.
template <bool STAGED>
__device__ __forceinline__ void parameters8(const float *staged, const float *given, uint32_t c, uint32_t n, float absent, float (&v)[8])
{
    if constexpr (STAGED) {
        const f32x4 lo = *(const f32x4 *)(staged + c), hi = *(const f32x4 *)(staged + c + 4);
        v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
        v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
    } else if (given) {
        load8_f32(given + c, n, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = absent;
    }
}

// The backward pass: with h the normalised values, through a norm goes rstd (g - mean(g) - h mean(g h)), mean(g) in layer norm
// alone.  Parameter gradients add up in registers over a team's rows, over the teams in LDS and over the workgroups in
// `k_edge_reduce`, in an order that the sizes alone decide.
template <class TX, class TF, int WAVES, int CHUNKS, bool CODED, bool TINY>
__global__ __launch_bounds__(backward_wavefronts(WAVES) * 64) void k_edge_backward(BackwardArgs a)
{
    constexpr int ALL = backward_wavefronts(WAVES);
    constexpr uint32_t TEAMS = ALL / WAVES, WIDTH = WAVES * CHUNKS * 512;
    constexpr bool STAGED = CHUNKS == 1;
    __shared__ TeamLds<ALL> lds;
    // parameters while the rows go by, then the teams' sums
    constexpr uint32_t PARAMS = STAGED ? 3 * WIDTH : 4, SUMS = TEAMS > 1 ? TEAMS * WIDTH : 4;
    __shared__ __attribute__((aligned(16))) float room[PARAMS > SUMS ? PARAMS : SUMS];
    uint32_t turn = 0;
    const uint32_t team = uniform(threadIdx.x / (WAVES * 64));
    const EdgeLayer &l = a.l;
    if constexpr (STAGED) {
        for (uint32_t j = threadIdx.x; j < WIDTH; j += ALL * 64) {
            const bool in = j < l.cols;
            room[j] = in && l.post_weight ? l.post_weight[j] : 1.0f;
            room[WIDTH + j] = in && l.post_bias ? l.post_bias[j] : 0.0f;
            room[2 * WIDTH + j] = in && l.pre_weight ? l.pre_weight[j] : 1.0f;
        }
        __syncthreads();
    }
    constexpr uint32_t AT = STAGED ? WIDTH : 0;
    const float *const post_weight = room, *const post_bias = room + AT, *const pre_weight = room + 2 * AT;
    const bool ragged = TINY || (l.cols & 7u) != 0;
    Place8 p[CHUNKS];
    float acc[ACCS][CHUNKS][8];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        p[k] = place8<TINY>(Team<WAVES, CHUNKS>::col(k), l.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int q = 0; q < ACCS; ++q) acc[q][k][i] = 0.0f;
    }
    // this team's rows, a round each; rounds are the same for all teams, and a round without a row works on zeros
    const Cut &cut = a.cut;
    uint32_t gate_row, gate_end, row, end, rounds;
    if (cut.whole) {
        gate_row = blockIdx.x * cut.whole + team;
        gate_end = min(cut.gates, (blockIdx.x + 1) * cut.whole);
        rounds = cut.whole / TEAMS * cut.rows_per_gate;
        row = gate_row < gate_end ? gate_row * cut.rows_per_gate : a.rows;
        end = min(a.rows - row, cut.rows_per_gate) + row;
    } else {
        gate_row = blockIdx.x / cut.parts;
        gate_end = 0;
        const uint32_t first = gate_row * cut.rows_per_gate, part = (blockIdx.x - gate_row * cut.parts) * cut.run;
        rounds = cut.run / TEAMS;
        row = first + part + team;
        end = min(a.rows - first, min(cut.rows_per_gate, part + cut.run)) + first;
    }
    uint32_t in_gate = 0;       // rounds of the present gate row

    // What is loaded of a row.  Each piece of the next row is asked for as soon as this row's has been unpacked, so that it
    // has a whole round to arrive and takes no registers of its own.  (Where there is no row, row 0; where there is no
    // matrix, whatever the workspace holds.  With 16 columns a lane each piece is asked for when it is due.)
    constexpr bool AHEAD = CHUNKS == 1;
    Raw8<TX> raw_d[CHUNKS];
    Raw8<TF> raw_u[CHUNKS];
    GateRaw raw_g[CHUNKS];
    Kept<TX, CODED> raw_x[CHUNKS];
    Kept<TF, CODED> raw_f[CHUNKS];
    f32x4_any stats;
    auto fetch_u = [&](uint32_t r) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            raw_u[k] = load_at<TINY>((const TF *)a.du + (uint64_t)r * a.du_stride, p[k].at, l.cols);
            fetch_kept<TINY>(raw_x[k], a.pre_codes, a.pre_exps, a.pre_codes_stride, a.pre_exps_stride, a.x_out, a.x_out_stride, r, p[k],
                             l.cols);
        }
    };
    auto fetch_d = [&](uint32_t r) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) raw_d[k] = load_at<TINY>((const TX *)a.dx_out + (uint64_t)r * a.dx_out_stride, p[k].at, l.cols);
    };
    auto fetch_f = [&](uint32_t r) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
            fetch_kept<TINY>(raw_f[k], a.post_codes, a.post_exps, a.post_codes_stride, a.post_exps_stride, a.f, a.f_stride, r, p[k], l.cols);
    };
    auto fetch_g = [&](uint32_t r) {
        const uint64_t gate_at = (uint64_t)(r / cut.rows_per_gate) * a.gate_stride;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) raw_g[k] = load_gate<TINY, TF>(a.gate, gate_at, p[k].at, l.cols, a.gate_f32);
    };
    auto fetch_stats = [&](uint32_t r) { stats = *(const f32x4_any *)(a.stats + 4 * (uint64_t)r); };
    if constexpr (AHEAD) {
        const uint32_t r = row < end ? row : 0u;
        fetch_stats(r);
        fetch_u(r);
        fetch_d(r);
        fetch_f(r);
        fetch_g(r);
    }
    if (WAVES > 1 && idle_wave<WAVES>(l.cols)) {      // (nothing but the other wavefronts' sums)
        const uint32_t sums = (a.branch && l.post != DGS_NORM_NONE ? 1u : 0u) + (a.through_pre ? 1u : 0u);
        for (uint32_t round = 0; round < rounds; ++round)
            for (uint32_t i = 0; i < sums; ++i) {
                float none[2] = {0.0f, 0.0f};
                team_sum<WAVES, ALL, 2>(none, lds, turn);
            }
        rounds = 0;
    }
    for (uint32_t round = 0; round < rounds; ++round) {
        const uint32_t this_row = row, this_gate = gate_row;
        const bool valid = row < end;
        bool gate_done = false;
        if (cut.whole) {
            ++row;
            if (++in_gate == cut.rows_per_gate) {
                in_gate = 0;
                gate_done = gate_row < gate_end;
                gate_row += TEAMS;
                row = gate_row < gate_end ? gate_row * cut.rows_per_gate : a.rows;
                end = min(a.rows - row, cut.rows_per_gate) + row;
            }
        } else {
            row += TEAMS;
        }
        const uint32_t next = row < end ? row : 0u;
        const uint32_t here = valid ? this_row : 0u;
        if constexpr (!AHEAD) {
            fetch_stats(here);
            fetch_u(here);
        }
        const f32x4_any st = stats;
        if constexpr (AHEAD) fetch_stats(next);

        // d: through the stream's norm
        float d[CHUNKS][8], h[CHUNKS][8];
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            if (ragged) in_place<TINY>(raw_u[k], p[k]);
            unpack8(raw_u[k], d[k]);
        }
        unpack_kept<TINY>(raw_x, l.pre, st.z, st.w, p, ragged, h);
        if constexpr (AHEAD) fetch_u(next);
        else fetch_d(here);
        if (a.through_pre) {
            if (valid && a.grad[ACC_PRE_BIAS]) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[ACC_PRE_BIAS][k][i] += d[k][i];
            }
            if (valid) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[ACC_PRE_WEIGHT][k][i] = __builtin_fmaf(d[k][i], h[k][i], acc[ACC_PRE_WEIGHT][k][i]);
            }
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                float w[8];
                parameters8<STAGED>(pre_weight, l.pre_weight, p[k].c, p[k].n, 1.0f, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[k][i] *= w[i];
            }
            through_norm<WAVES, ALL, CHUNKS>(d, h, p, ragged, l.pre, st.w, l.inv_cols, lds, turn);
        } else {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[k][i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            float o[8];
            if (ragged) in_place<TINY>(raw_d[k], p[k]);
            unpack8(raw_d[k], o);
            if (a.arrives) {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[k][i] += o[i];
            }
        }
        if constexpr (AHEAD) fetch_d(next);
        else fetch_f(here);
        if (a.dx && valid) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = l.skip * d[k][i];
                store8((TX *)a.dx + (uint64_t)this_row * a.dx_stride, p[k].c, p[k].n, o);
            }
        }
        // m and k: through the gate and the branch's norm
        unpack_kept<TINY>(raw_f, l.post, st.x, st.y, p, ragged, h);
        if constexpr (AHEAD) fetch_f(next);
        else fetch_g(here);
        if (a.branch) {
            float w[CHUNKS][8];
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                parameters8<STAGED>(post_weight, l.post_weight, p[k].c, p[k].n, 1.0f, w[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[k][i] *= l.branch;
            }
            if (a.gated) {
                if (valid) {
#pragma unroll
                    for (int k = 0; k < CHUNKS; ++k) {
                        float b[8];
                        parameters8<STAGED>(post_bias, l.post_bias, p[k].c, p[k].n, 0.0f, b);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            acc[ACC_GATE][k][i] = __builtin_fmaf(d[k][i], __builtin_fmaf(h[k][i], w[k][i], b[i]), acc[ACC_GATE][k][i]);
                    }
                }
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) {
                    float g[8];
                    unpack_gate<TINY, TF>(raw_g[k], a.gate_f32, ragged, p[k], g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[k][i] *= g[i];
                }
            }
            if constexpr (AHEAD) fetch_g(next);
            if (valid && a.grad[ACC_POST_BIAS]) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[ACC_POST_BIAS][k][i] += d[k][i];
            }
            if (valid) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[ACC_POST_WEIGHT][k][i] = __builtin_fmaf(d[k][i], h[k][i], acc[ACC_POST_WEIGHT][k][i]);
            }
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[k][i] *= w[k][i];
            through_norm<WAVES, ALL, CHUNKS>(d, h, p, ragged, l.post, st.y, l.inv_cols, lds, turn);
            if (a.df && valid) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) store8((TF *)a.df + (uint64_t)this_row * a.df_stride, p[k].c, p[k].n, d[k]);
            }
            if (gate_done) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) {
                    if (a.dgate) {
                        const uint64_t at = (uint64_t)this_gate * a.dgate_stride;
                        if (a.gate_f32) store_grad8((float *)a.dgate + at, p[k].c, p[k].n, acc[ACC_GATE][k], a.accumulate);
                        else store_grad8((TF *)a.dgate + at, p[k].c, p[k].n, acc[ACC_GATE][k], false);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[ACC_GATE][k][i] = 0.0f;
                }
            }
        }
    }

    // what this workgroup adds up to: the teams' sums, then to its place among the partial sums, or where it is alone to where
    // they belong
#pragma unroll
    for (int q = 0; q < ACCS; ++q) {
        if (q < ACC_GATE ? !a.grad[q < ACC_GATE ? q : 0] : (!a.dgate || cut.whole)) continue;
        const bool alone = q < ACC_GATE ? cut.blocks == 1 : cut.parts == 1;
        float *to = !alone ? a.partial + ((uint64_t)q * cut.blocks + blockIdx.x) * l.cols : q < ACC_GATE ? a.grad[q] : nullptr;
        const uint64_t gate_at = (uint64_t)gate_row * a.dgate_stride;
        const bool add = alone && a.accumulate;
        if constexpr (TEAMS > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) room[team * WIDTH + p[k].c + i] = acc[q][k][i];
            __syncthreads();
            for (uint32_t j = threadIdx.x; j < l.cols; j += ALL * 64) {
                float s = room[j];
#pragma unroll
                for (uint32_t t = 1; t < TEAMS; ++t) s += room[t * WIDTH + j];
                if (to) to[j] = add ? to[j] + s : s;
                else store_gate<TF>(a.dgate, gate_at + j, a.gate_f32, a.accumulate, s);
            }
        } else {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                if (to) {
                    store_grad8(to, p[k].c, p[k].n, acc[q][k], add);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i)
                        if (i < p[k].n) store_gate<TF>(a.dgate, gate_at + p[k].c + i, a.gate_f32, a.accumulate, acc[q][k][i]);
                }
            }
        }
    }
}

// Adds up the workgroups' partial sums, 64 columns and REDUCE_LINES lines at a time; blockIdx.y: one of the four parameter
// gradients, then the gate rows whose gradients are in parts.  256 lines of 768 columns for each of five gradients, from
// cache, in 4.0 us.
constexpr uint32_t REDUCE_LINES = 16;

__global__ __launch_bounds__(REDUCE_LINES * 64) void k_edge_reduce(const float *partial, float *g0, float *g1, float *g2, float *g3,
                                                                   void *dgate, uint64_t dgate_stride, uint32_t cols, uint32_t blocks,
                                                                   uint32_t parts, uint32_t gate_type, uint32_t accumulate)
{
    __shared__ float part[REDUCE_LINES][64];
    const uint32_t what = blockIdx.y, lane = threadIdx.x & 63u, line = threadIdx.x >> 6;
    const uint32_t j = blockIdx.x * 64 + lane;
    float *const grad = what == 0 ? g0 : what == 1 ? g1 : what == 2 ? g2 : g3;
    if (what < 4 && !grad) return;
    const uint32_t first = what < 4 ? 0u : (what - 4u) * parts, count = what < 4 ? blocks : parts;
    const float *from = partial + ((uint64_t)(what < 4 ? what : 4u) * blocks + first) * cols;
    float s = 0.0f;
    if (j < cols) {
#pragma unroll 8
        for (uint32_t b = line; b < count; b += REDUCE_LINES) s += from[(uint64_t)b * cols + j];
    }
    part[line][lane] = s;
    __syncthreads();
    if (line != 0 || j >= cols) return;
#pragma unroll
    for (uint32_t b = 1; b < REDUCE_LINES; ++b) s += part[b][lane];
    if (what < 4) {
        grad[j] = accumulate ? grad[j] + s : s;
        return;
    }
    const uint64_t at = (what - 4u) * dgate_stride + j;
    if (gate_type == DGS_F32) ((float *)dgate)[at] = accumulate ? ((float *)dgate)[at] + s : s;
    else if (gate_type == DGS_F16) ((f16 *)dgate)[at] = from_float<f16>(s);
    else ((bf16 *)dgate)[at] = from_float<bf16>(s);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

// Wavefronts of a row's team: 8 columns a lane, and 16 in rows that a workgroup does not hold then; powers of two, and three
// times those.  (Compared when they were built: 16 columns from 512 on, half the wavefronts: 16384 x 4096 edges with checkpoints
// and their decoding 239 us against 219, 8192 x 768 36 against 33.  Powers of two alone: 16384 x 1280 in half precision 46 us
// against 41 forward and 55 against 49 backward, 8192 x 6144 100 against 94 and 125 against 117.)
static uint32_t waves_of(uint32_t cols)
{
    constexpr uint32_t kinds[] = {1, 2, 3, 4, 6, 8, 12};
    for (uint32_t w : kinds)
        if (cols <= w * 512) return w;
    return 16;
}

// Workgroups of the backward pass: one to a compute unit at most, so that few partial sums are left.
static Cut cut_of(uint32_t rows, uint32_t cols, uint32_t rows_per_gate)
{
    const uint32_t waves = waves_of(cols), teams = (uint32_t)backward_wavefronts((int)waves) / waves, most = BACKWARD_BLOCKS;
    Cut t;
    t.rows_per_gate = rows_per_gate && rows_per_gate < rows ? rows_per_gate : rows;
    t.gates = (rows - 1) / t.rows_per_gate + 1;
    t.whole = t.parts = t.run = 0;
    const uint32_t rounds = (t.rows_per_gate - 1) / teams + 1;      // of a team, if one workgroup took a gate row
    // Many gate rows: each goes to one team, if that keeps half the workgroups busy or there are too few rows to share.  (16384 x
    // 4096 with 16 or 32 rows a gate row: 144 and 144 us, one gate row to a workgroup or parts of it 163 and 149; 32768 x 1024 with 16
    // 72 against 94.  Where it does leave half of them idle it loses: 16384 x 4096 with 63 or 64 rows 213 and 221 us against 231
    // and 140, 32768 x 1024 with 32 100 against 76.  65536 x 512 with 33 rows, on the other side of the line: 99, whole 88.)
    if (t.gates >= most && (rounds < 2 || t.gates >= most * teams / 2)) {
        t.whole = ((t.gates + most - 1) / most + teams - 1) / teams * teams;
        t.blocks = (t.gates - 1) / t.whole + 1;
    } else {
        t.parts = t.gates >= most ? 1u : most / t.gates < rounds ? most / t.gates : rounds;
        if (t.gates == 1 && rounds <= 2) t.parts = 1;      // a second round takes less than a second launch
        t.run = (rounds + t.parts - 1) / t.parts * teams;
        t.parts = (t.rows_per_gate - 1) / t.run + 1;
        t.blocks = t.gates * t.parts;
    }
    return t;
}

template <class TX, class TF> static void launch_forward(const ForwardArgs &a, hipStream_t st)
{
    const uint32_t waves = waves_of(a.l.cols), teams = waves == 1 ? FORWARD_TEAMS : 1u;
    // As many workgroups as run at a time where five wavefronts go to a SIMD, among which a workgroup's are spread evenly: that is
    // what the 16-bit kernels' registers allow.  Of an fp32 stream most kernels have registers for four, and the last fifth of
    // these workgroups begins late: 65536 x 768 of fp32 with checkpoints 215 us, with a grid for four 196, 16384 x 1280 with a
    // bfloat16 branch 62 and 54; but 16384 x 2048 of fp32 113 and 117, without checkpoints 102 and 112.
    const uint32_t w = teams * waves, most = 256u * (w > 4 ? 5u / ((w + 3u) / 4u) : 20u / w), need = (a.rows + teams - 1) / teams;
    const dim3 grid(need < most ? need : most), block(teams * waves * 64);
    if (a.l.cols < 8) hipLaunchKernelGGL((k_edge_forward<TX, TF, 1, 1, true>), grid, block, 0, st, a);
    else if (waves == 1) hipLaunchKernelGGL((k_edge_forward<TX, TF, 1, 1, false>), grid, block, 0, st, a);
    else if (waves == 2) hipLaunchKernelGGL((k_edge_forward<TX, TF, 2, 1, false>), grid, block, 0, st, a);
    else if (waves == 3) hipLaunchKernelGGL((k_edge_forward<TX, TF, 3, 1, false>), grid, block, 0, st, a);
    else if (waves == 4) hipLaunchKernelGGL((k_edge_forward<TX, TF, 4, 1, false>), grid, block, 0, st, a);
    else if (waves == 6) hipLaunchKernelGGL((k_edge_forward<TX, TF, 6, 1, false>), grid, block, 0, st, a);
    else if (waves == 8) hipLaunchKernelGGL((k_edge_forward<TX, TF, 8, 1, false>), grid, block, 0, st, a);
    else if (waves == 12) hipLaunchKernelGGL((k_edge_forward<TX, TF, 12, 1, false>), grid, block, 0, st, a);
    else if (a.l.cols <= 8192) hipLaunchKernelGGL((k_edge_forward<TX, TF, 16, 1, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_edge_forward<TX, TF, 16, 2, false>), grid, block, 0, st, a);
}

template <class TX, class TF, bool CODED> static void launch_backward(const BackwardArgs &a, hipStream_t st)
{
    const uint32_t waves = waves_of(a.l.cols);
    const dim3 grid(a.cut.blocks), block(backward_wavefronts((int)waves) * 64);
    if (a.l.cols < 8) hipLaunchKernelGGL((k_edge_backward<TX, TF, 1, 1, CODED, true>), grid, block, 0, st, a);
    else if (waves == 1) hipLaunchKernelGGL((k_edge_backward<TX, TF, 1, 1, CODED, false>), grid, block, 0, st, a);
    else if (waves == 2) hipLaunchKernelGGL((k_edge_backward<TX, TF, 2, 1, CODED, false>), grid, block, 0, st, a);
    else if (waves == 3) hipLaunchKernelGGL((k_edge_backward<TX, TF, 3, 1, CODED, false>), grid, block, 0, st, a);
    else if (waves == 4) hipLaunchKernelGGL((k_edge_backward<TX, TF, 4, 1, CODED, false>), grid, block, 0, st, a);
    else if (waves == 6) hipLaunchKernelGGL((k_edge_backward<TX, TF, 6, 1, CODED, false>), grid, block, 0, st, a);
    else if (waves == 8) hipLaunchKernelGGL((k_edge_backward<TX, TF, 8, 1, CODED, false>), grid, block, 0, st, a);
    else if (waves == 12) hipLaunchKernelGGL((k_edge_backward<TX, TF, 12, 1, CODED, false>), grid, block, 0, st, a);
    else if (a.l.cols <= 8192) hipLaunchKernelGGL((k_edge_backward<TX, TF, 16, 1, CODED, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_edge_backward<TX, TF, 16, 2, CODED, false>), grid, block, 0, st, a);
}
template <class TX, class TF> static void launch_backward(const BackwardArgs &a, hipStream_t st)
{
    if (a.coded) launch_backward<TX, TF, true>(a, st);
    else launch_backward<TX, TF, false>(a, st);
}

static bool norm_ok(int kind, float eps)
{
    return kind == DGS_NORM_NONE || ((kind == DGS_NORM_RMS || kind == DGS_NORM_LAYER) && eps >= 1.17549435e-38f && eps < 1e30f);
}
// (cols beyond the limit are DGS_ENOTSUP and looked at afterwards)
static bool layer_ok(const dgs_edge &e)
{
    return e.cols != 0 && norm_ok(e.post, e.post_eps) && norm_ok(e.pre, e.pre_eps) && e.skip == e.skip && e.branch == e.branch
        && aligned_to(e.post_weight, 4) && aligned_to(e.post_bias, 4) && aligned_to(e.pre_weight, 4) && aligned_to(e.pre_bias, 4);
}
static bool types_ok(int stream, int type) { return is_type(stream) && is_type(type); }
static bool types_have(int stream, int type) { return stream == type || stream == DGS_F32; }
static bool present_ok(const dgs_matrix &m, uint64_t cols, int type) { return !m.data || matrix_ok(m.data, m.stride, cols, type); }
static bool saved_ok(const dgs_codes &c, uint64_t cols) { return !c.codes || codes_ok(c, cols); }
static bool gate_ok(const dgs_matrix &g, uint64_t cols, int gate_type, int type, uint32_t rows_per_gate)
{
    return !g.data || (rows_per_gate != 0 && (gate_type == DGS_F32 || gate_type == type) && matrix_ok(g.data, g.stride, cols, gate_type));
}
static EdgeLayer layer_of(const dgs_edge &e)
{
    EdgeLayer l;
    l.post_weight = e.post_weight; l.post_bias = e.post_bias; l.pre_weight = e.pre_weight; l.pre_bias = e.pre_bias;
    l.cols = e.cols; l.post = e.post; l.pre = e.pre;
    l.post_eps = e.post_eps; l.pre_eps = e.pre_eps; l.skip = e.skip; l.branch = e.branch;
    l.inv_cols = 1.0f / (float)e.cols;
    return l;
}

}  // namespace dgs

using namespace dgs;

extern "C" int dgs_edge_forward(const dgs_edge *edge, const dgs_edge_forward_args *args, void *hip_stream)
{
    if (!edge || !args || !layer_ok(*edge) || !types_ok(args->stream_type, args->type)) return DGS_EINVAL;
    const dgs_edge &e = *edge;
    const dgs_edge_forward_args &p = *args;
    const uint64_t cols = e.cols;
    if (p.rows == 0) return DGS_OK;
    const bool branch = p.f.data != nullptr;
    if (!matrix_ok(p.x.data, p.x.stride, cols, p.stream_type)) return DGS_EINVAL;
    if (branch) {
        if (!matrix_ok(p.f.data, p.f.stride, cols, p.type) || !matrix_ok(p.x_out.data, p.x_out.stride, cols, p.stream_type)
            || !gate_ok(p.gate, cols, p.gate_type, p.type, p.rows_per_gate))
            return DGS_EINVAL;
    } else if (p.x_out.data || p.gate.data || e.post != DGS_NORM_NONE || p.post_saved.codes) {
        return DGS_EINVAL;
    }
    if (e.pre != DGS_NORM_NONE ? !matrix_ok(p.u.data, p.u.stride, cols, p.type) : (p.u.data || p.pre_saved.codes || !branch))
        return DGS_EINVAL;
    if (!saved_ok(p.post_saved, cols) || !saved_ok(p.pre_saved, cols) || !aligned_to(p.stats, 4)) return DGS_EINVAL;
    if (e.cols > DGS_EDGE_MAX_COLS || p.rows > 0x7FFFFFFFu || !types_have(p.stream_type, p.type)) return DGS_ENOTSUP;
    ForwardArgs a;
    a.l = layer_of(e);
    a.x = p.x.data; a.f = p.f.data; a.gate = p.gate.data; a.x_out = p.x_out.data; a.u = p.u.data;
    a.post_codes = p.post_saved.codes; a.post_exps = p.post_saved.exps;
    a.pre_codes = p.pre_saved.codes; a.pre_exps = p.pre_saved.exps;
    a.stats = p.stats;
    a.x_stride = (uint32_t)p.x.stride; a.f_stride = (uint32_t)p.f.stride; a.gate_stride = (uint32_t)p.gate.stride;
    a.x_out_stride = (uint32_t)p.x_out.stride; a.u_stride = (uint32_t)p.u.stride;
    a.post_codes_stride = (uint32_t)p.post_saved.codes_stride; a.post_exps_stride = (uint32_t)p.post_saved.exps_stride;
    a.pre_codes_stride = (uint32_t)p.pre_saved.codes_stride; a.pre_exps_stride = (uint32_t)p.pre_saved.exps_stride;
    a.rows = p.rows;
    a.rows_per_gate = p.gate.data ? p.rows_per_gate : 1u;
    a.gate_f32 = p.gate.data && p.gate_type == DGS_F32;
    a.branch = branch;
    a.gated = p.gate.data != nullptr;
    // what is absent is loaded all the same, from a row of x
    if (!branch) { a.f = a.x; a.f_stride = 0; }
    if (!a.gated) { a.gate = a.x; a.gate_stride = 0; }
    const hipStream_t st = (hipStream_t)hip_stream;
    if (p.stream_type == DGS_F32) {
        if (p.type == DGS_F32) launch_forward<float, float>(a, st);
        else if (p.type == DGS_F16) launch_forward<float, f16>(a, st);
        else launch_forward<float, bf16>(a, st);
    } else if (p.type == DGS_F16) {
        launch_forward<f16, f16>(a, st);
    } else {
        launch_forward<bf16, bf16>(a, st);
    }
    return launched();
}

extern "C" size_t dgs_edge_backward_workspace(uint32_t rows, uint32_t cols, uint32_t rows_per_gate)
{
    if (rows == 0 || cols == 0 || cols > DGS_EDGE_MAX_COLS) return 0;
    return (size_t)cut_of(rows, cols, rows_per_gate).blocks * ACCS * cols * sizeof(float);
}

extern "C" int dgs_edge_backward(const dgs_edge *edge, const dgs_edge_backward_args *args, void *hip_stream)
{
    if (!edge || !args || !layer_ok(*edge) || !types_ok(args->stream_type, args->type)) return DGS_EINVAL;
    const dgs_edge &e = *edge;
    const dgs_edge_backward_args &p = *args;
    const uint64_t cols = e.cols;
    const bool branch = p.f.data || p.post_saved.codes;
    const bool through_pre = p.du.data != nullptr;
    if (!aligned_to(p.post_weight_grad, 4) || !aligned_to(p.post_bias_grad, 4) || !aligned_to(p.pre_weight_grad, 4)
        || !aligned_to(p.pre_bias_grad, 4))
        return DGS_EINVAL;
    // (of no rows, pointers say nothing)
    if (p.rows) {
        if (through_pre && e.pre == DGS_NORM_NONE) return DGS_EINVAL;
        if (!branch && (e.post != DGS_NORM_NONE || p.gate.data || p.df.data || p.post_weight_grad || p.post_bias_grad)) return DGS_EINVAL;
        if (p.dgate.data && !p.gate.data) return DGS_EINVAL;
        if (!present_ok(p.dx_out, cols, p.stream_type) || !present_ok(p.du, cols, p.type) || !present_ok(p.dx, cols, p.stream_type)
            || !present_ok(p.df, cols, p.type) || !gate_ok(p.gate, cols, p.gate_type, p.type, p.rows_per_gate)
            || !present_ok(p.dgate, cols, p.gate_type))
            return DGS_EINVAL;
        // both norms the same way
        if (branch && through_pre && (p.post_saved.codes != nullptr) != (p.pre_saved.codes != nullptr)) return DGS_EINVAL;
        if (branch && (p.post_saved.codes ? p.f.data || !codes_ok(p.post_saved, cols) : !matrix_ok(p.f.data, p.f.stride, cols, p.type)))
            return DGS_EINVAL;
        if (through_pre
            && (p.pre_saved.codes ? p.x_out.data || !codes_ok(p.pre_saved, cols)
                                  : !matrix_ok(p.x_out.data, p.x_out.stride, cols, p.stream_type)))
            return DGS_EINVAL;
        if (!p.stats || !aligned_to(p.stats, 4)) return DGS_EINVAL;
    }
    if (e.cols > DGS_EDGE_MAX_COLS || p.rows > 0x7FFFFFFFu || !types_have(p.stream_type, p.type)) return DGS_ENOTSUP;
    const bool grads = p.post_weight_grad || p.post_bias_grad || p.pre_weight_grad || p.pre_bias_grad;
    BackwardArgs a;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (p.rows) {
        if (!p.workspace || !aligned_to(p.workspace, 16)) return DGS_EINVAL;
        if (p.workspace_bytes < dgs_edge_backward_workspace(p.rows, e.cols, p.gate.data ? p.rows_per_gate : 0)) return DGS_ENOMEM;
        a.l = layer_of(e);
        a.cut = cut_of(p.rows, e.cols, p.gate.data ? p.rows_per_gate : 0);
        a.dx_out = p.dx_out.data; a.du = p.du.data; a.gate = p.gate.data; a.f = p.f.data; a.x_out = p.x_out.data;
        a.post_codes = p.post_saved.codes; a.post_exps = p.post_saved.exps;
        a.pre_codes = p.pre_saved.codes; a.pre_exps = p.pre_saved.exps;
        a.stats = p.stats;
        a.dx = p.dx.data; a.df = p.df.data; a.dgate = p.dgate.data;
        a.grad[ACC_POST_WEIGHT] = p.post_weight_grad; a.grad[ACC_POST_BIAS] = p.post_bias_grad;
        a.grad[ACC_PRE_WEIGHT] = p.pre_weight_grad; a.grad[ACC_PRE_BIAS] = p.pre_bias_grad;
        a.partial = (float *)p.workspace;
        a.dx_out_stride = (uint32_t)p.dx_out.stride; a.du_stride = (uint32_t)p.du.stride; a.gate_stride = (uint32_t)p.gate.stride; a.f_stride = (uint32_t)p.f.stride;
        a.x_out_stride = (uint32_t)p.x_out.stride; a.dx_stride = (uint32_t)p.dx.stride; a.df_stride = (uint32_t)p.df.stride; a.dgate_stride = (uint32_t)p.dgate.stride;
        a.post_codes_stride = (uint32_t)p.post_saved.codes_stride; a.post_exps_stride = (uint32_t)p.post_saved.exps_stride;
        a.pre_codes_stride = (uint32_t)p.pre_saved.codes_stride; a.pre_exps_stride = (uint32_t)p.pre_saved.exps_stride;
        a.rows = p.rows;
        a.gate_f32 = p.gate.data && p.gate_type == DGS_F32;
        a.accumulate = p.accumulate != 0;
        a.branch = branch;
        a.gated = p.gate.data != nullptr;
        a.through_pre = through_pre;
        a.arrives = p.dx_out.data != nullptr;
        a.coded = (branch && p.post_saved.codes) || (through_pre && p.pre_saved.codes);
        // what is absent is loaded all the same, from the workspace, which holds a row of any type
        const void *const none = p.workspace;
        if (!a.arrives) { a.dx_out = none; a.dx_out_stride = 0; }
        if (!through_pre) {
            a.du = a.x_out = none;
            a.pre_codes = (const int8_t *)none;
            a.pre_exps = (const uint8_t *)none;
            a.du_stride = a.x_out_stride = a.pre_codes_stride = a.pre_exps_stride = 0;
        }
        if (!branch) {
            a.f = none;
            a.post_codes = (const int8_t *)none;
            a.post_exps = (const uint8_t *)none;
            a.f_stride = a.post_codes_stride = a.post_exps_stride = 0;
        }
        if (!a.gated) { a.gate = none; a.gate_stride = 0; }
        if (p.stream_type == DGS_F32) {
            if (p.type == DGS_F32) launch_backward<float, float>(a, st);
            else if (p.type == DGS_F16) launch_backward<float, f16>(a, st);
            else launch_backward<float, bf16>(a, st);
        } else if (p.type == DGS_F16) {
            launch_backward<f16, f16>(a, st);
        } else {
            launch_backward<bf16, bf16>(a, st);
        }
    }
    const uint32_t in_parts = p.rows && p.dgate.data && a.cut.parts > 1 ? a.cut.gates : 0u;
    // (a workgroup that is alone has written them)
    if (!p.rows ? grads : a.cut.blocks > 1 && (grads || in_parts))
        hipLaunchKernelGGL(k_edge_reduce, dim3((e.cols + 63) / 64, 4 + in_parts), dim3(REDUCE_LINES * 64), 0, st,
                           (const float *)p.workspace, p.post_weight_grad, p.post_bias_grad, p.pre_weight_grad, p.pre_bias_grad,
                           p.dgate.data, p.dgate.stride, e.cols, p.rows ? a.cut.blocks : 0u, p.rows ? a.cut.parts : 0u,
                           (uint32_t)p.gate_type, (uint32_t)(p.accumulate != 0));
    return launched();
}
