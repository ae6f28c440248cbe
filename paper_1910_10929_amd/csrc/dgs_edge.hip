// The edge between two blocks: norm of the branch, gate, residual sum and norm of the stream in one pass over the rows, and
// its gradients in another.
//
// A row belongs to a team of wavefronts that holds all of it in registers, eight consecutive columns in a lane, so that the
// statistics are taken of what is there (mean first, then the squares of what is left) and every matrix is read and written
// once.  Parameters stay in registers from row to row, and the next row's loads are issued before a row is worked on.
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
    uint64_t x_stride, f_stride, gate_stride, x_out_stride, u_stride;
    uint64_t post_codes_stride, post_exps_stride, pre_codes_stride, pre_exps_stride;
    uint32_t rows, rows_per_gate, gate_f32;
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

// A gate's eight values: fp32, or of the branch's type.
struct GateRaw { uint32_t w[8]; };
template <class TF> __device__ __forceinline__ GateRaw load_gate(const void *gate, uint64_t at, uint32_t n, bool f32)
{
    GateRaw g;
    if (f32) {
        const Raw8<float> r = load8((const float *)gate + at, n);
        __builtin_memcpy(&g, &r, sizeof(r));
    } else {
        const Raw8<TF> r = load8((const TF *)gate + at, n);
        __builtin_memcpy(&g, &r, sizeof(r));
    }
    return g;
}
template <class TF> __device__ __forceinline__ void unpack_gate(const GateRaw &g, bool f32, float (&v)[8])
{
    if (f32) {
        Raw8<float> r;
        __builtin_memcpy(&r, &g, sizeof(r));
        unpack8(r, v);
    } else {
        Raw8<TF> r;
        __builtin_memcpy(&r, &g, sizeof(r));
        unpack8(r, v);
    }
}

// Wavefronts of a workgroup whose teams are single wavefronts.
constexpr uint32_t FORWARD_TEAMS = 4, BACKWARD_TEAMS = 8;

template <int WAVES, int CHUNKS> struct Team {
    static constexpr uint32_t LANES = WAVES * 64;
    // first column of this lane's k-th eight
    static __device__ __forceinline__ uint32_t col(int k) { return ((uint32_t)k * LANES + threadIdx.x % LANES) * 8u; }
};

// Statistics of a row and its normalised values, in place.
template <int WAVES, int CHUNKS>
__device__ __forceinline__ void normalise(float (&v)[CHUNKS][8], const uint32_t (&n)[CHUNKS], int kind, float eps, float inv_cols,
                                          float (*lds)[2][WAVES], uint32_t &turn, float &mean, float &rstd)
{
    mean = rstd = 0.0f;
    if (kind == DGS_NORM_NONE) return;
    float s[1];
    if (kind == DGS_NORM_LAYER) {
        s[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += v[k][i];
        team_sum<WAVES, 1>(s, lds, turn);
        mean = s[0] * inv_cols;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = (uint32_t)i < n[k] ? v[k][i] - mean : 0.0f;
    }
    s[0] = 0.0f;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = __builtin_fmaf(v[k][i], v[k][i], s[0]);
    team_sum<WAVES, 1>(s, lds, turn);
    rstd = rsqrt_of(__builtin_fmaf(s[0], inv_cols, eps));
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] *= rstd;
}

template <class TX, class TF, int CHUNKS> struct ForwardRow {
    Raw8<TX> x[CHUNKS];
    Raw8<TF> f[CHUNKS];
    GateRaw g[CHUNKS];
};

template <class TX, class TF, int WAVES, int CHUNKS>
__device__ __forceinline__ void fetch(ForwardRow<TX, TF, CHUNKS> &r, const ForwardArgs &a, uint32_t row, const uint32_t (&c)[CHUNKS],
                                      const uint32_t (&n)[CHUNKS])
{
    const uint64_t gate_at = a.gate ? (uint64_t)(row / a.rows_per_gate) * a.gate_stride : 0u;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        r.x[k] = load8((const TX *)a.x + row * a.x_stride + c[k], n[k]);
        if (a.f) r.f[k] = load8((const TF *)a.f + row * a.f_stride + c[k], n[k]);
        if (a.gate) r.g[k] = load_gate<TF>(a.gate, gate_at + c[k], n[k], a.gate_f32);
    }
}

template <class TX, class TF, int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES == 1 ? FORWARD_TEAMS * 64 : WAVES * 64) void k_edge_forward(ForwardArgs a)
{
    constexpr uint32_t TEAMS = WAVES == 1 ? FORWARD_TEAMS : 1;
    __shared__ float lds[2][2][WAVES];
    uint32_t turn = 0;
    const uint32_t team = uniform(blockIdx.x * TEAMS + threadIdx.x / (WAVES * 64));
    const uint32_t teams = gridDim.x * TEAMS;
    const EdgeLayer &l = a.l;
    uint32_t c[CHUNKS], n[CHUNKS];
    float wp[CHUNKS][8], bp[CHUNKS][8], wn[CHUNKS][8], bn[CHUNKS][8];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        c[k] = Team<WAVES, CHUNKS>::col(k);
        n[k] = live8(c[k], l.cols);
        if (l.post_weight) load8_f32(l.post_weight + c[k], n[k], wp[k]);
        if (l.post_bias) load8_f32(l.post_bias + c[k], n[k], bp[k]);
        if (l.pre_weight) load8_f32(l.pre_weight + c[k], n[k], wn[k]);
        if (l.pre_bias) load8_f32(l.pre_bias + c[k], n[k], bn[k]);
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
    ForwardRow<TX, TF, CHUNKS> next;
    fetch<TX, TF, WAVES, CHUNKS>(next, a, row, c, n);
    for (; row < a.rows; row += teams) {
        const ForwardRow<TX, TF, CHUNKS> now = next;
        if (row + teams < a.rows) fetch<TX, TF, WAVES, CHUNKS>(next, a, row + teams, c, n);
        float x[CHUNKS][8], f[CHUNKS][8];
        float post_mean = 0.0f, post_rstd = 0.0f, pre_mean, pre_rstd;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) unpack8(now.x[k], x[k]);
        if (a.f) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) unpack8(now.f[k], f[k]);
            normalise<WAVES, CHUNKS>(f, n, l.post, l.post_eps, l.inv_cols, lds, turn, post_mean, post_rstd);
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                if (a.post_codes)
                    save8(a.post_codes + row * a.post_codes_stride, a.post_exps + row * a.post_exps_stride, c[k], n[k], f[k]);
                float g[8];
                if (a.gate) unpack_gate<TF>(now.g[k], a.gate_f32, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float m = a.gate ? l.branch * g[i] : l.branch;
                    x[k][i] = __builtin_fmaf(m, __builtin_fmaf(f[k][i], wp[k][i], bp[k][i]), l.skip * x[k][i]);
                }
                store8((TX *)a.x_out + row * a.x_out_stride + c[k], n[k], x[k]);
            }
        }
        normalise<WAVES, CHUNKS>(x, n, l.pre, l.pre_eps, l.inv_cols, lds, turn, pre_mean, pre_rstd);
        if (l.pre != DGS_NORM_NONE) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                if (a.pre_codes)
                    save8(a.pre_codes + row * a.pre_codes_stride, a.pre_exps + row * a.pre_exps_stride, c[k], n[k], x[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[k][i] = __builtin_fmaf(x[k][i], wn[k][i], bn[k][i]);
                store8((TF *)a.u + row * a.u_stride + c[k], n[k], x[k]);
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

// How rows are dealt out to workgroups.  Where gate rows are few, every gate row's rows are cut into `parts` runs of `run`
// rows, one per workgroup, and the parts of its gradient are added up afterwards; where they are many, a workgroup takes
// `whole` gate rows and writes their gradients itself.
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
    uint64_t dx_out_stride, du_stride, gate_stride, f_stride, x_out_stride, dx_stride, df_stride, dgate_stride;
    uint64_t post_codes_stride, post_exps_stride, pre_codes_stride, pre_exps_stride;
    uint32_t rows, gate_f32, accumulate, branch;     // branch: there is one
};

enum { ACC_POST_WEIGHT, ACC_POST_BIAS, ACC_PRE_WEIGHT, ACC_PRE_BIAS, ACC_GATE, ACCS };

// Normalised values as the forward pass left them: codes, or the values themselves.
template <class T> struct Kept { Raw8<T> v; uint32_t q[2]; uint32_t byte; };

template <class T>
__device__ __forceinline__ void fetch_kept(Kept<T> &r, const int8_t *codes, const uint8_t *exps, uint64_t codes_stride,
                                           uint64_t exps_stride, const void *values, uint64_t stride, uint64_t row, uint32_t c, uint32_t n)
{
    if (codes) {
        load_codes(codes + row * codes_stride + c, n, r.q);
        r.byte = n ? exps[row * exps_stride + c / DGS_CHECKPOINT_RUN] : 1u;
    } else {
        r.v = load8((const T *)values + row * stride + c, n);
    }
}
template <class T>
__device__ __forceinline__ void unpack_kept(const Kept<T> &r, bool coded, int kind, float mean, float rstd, uint32_t n, float (&v)[8])
{
    if (coded) {
        decode8(r.q, run_scale(r.byte), v);
        return;
    }
    unpack8(r.v, v);
    if (kind == DGS_NORM_NONE) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (uint32_t)i < n ? (v[i] - mean) * rstd : 0.0f;
}

template <class TX, class TF, int CHUNKS> struct BackwardRow {
    Raw8<TX> d[CHUNKS];
    Raw8<TF> u[CHUNKS];
    GateRaw g[CHUNKS];
    Kept<TF> f[CHUNKS];
    Kept<TX> x[CHUNKS];
    f32x4_any stats;
};

template <class TX, class TF, int WAVES, int CHUNKS>
__device__ __forceinline__ void fetch(BackwardRow<TX, TF, CHUNKS> &r, const BackwardArgs &a, uint32_t row, const uint32_t (&c)[CHUNKS],
                                      const uint32_t (&n)[CHUNKS])
{
    const uint64_t gate_at = a.gate ? (uint64_t)(row / a.cut.rows_per_gate) * a.gate_stride : 0u;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        if (a.dx_out) r.d[k] = load8((const TX *)a.dx_out + row * a.dx_out_stride + c[k], n[k]);
        if (a.du) {
            r.u[k] = load8((const TF *)a.du + row * a.du_stride + c[k], n[k]);
            fetch_kept<TX>(r.x[k], a.pre_codes, a.pre_exps, a.pre_codes_stride, a.pre_exps_stride, a.x_out, a.x_out_stride, row, c[k],
                           n[k]);
        }
        if (a.branch)
            fetch_kept<TF>(r.f[k], a.post_codes, a.post_exps, a.post_codes_stride, a.post_exps_stride, a.f, a.f_stride, row, c[k], n[k]);
        if (a.gate) r.g[k] = load_gate<TF>(a.gate, gate_at + c[k], n[k], a.gate_f32);
    }
    r.stats = *(const f32x4_any *)(a.stats + 4 * (uint64_t)row);
}

// The gradient through a norm at its normalised output h, times rstd: in place.  Columns beyond the row hold 0 in g and h and
// are not read of the result.
template <int WAVES, int CHUNKS>
__device__ __forceinline__ void through_norm(float (&g)[CHUNKS][8], const float (&h)[CHUNKS][8], int kind, float rstd, float inv_cols,
                                             float (*lds)[2][WAVES], uint32_t &turn)
{
    if (kind == DGS_NORM_NONE) return;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = __builtin_fmaf(g[k][i], h[k][i], s[0]);
    if (kind == DGS_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[1] += g[k][i];
    }
    team_sum<WAVES, 2>(s, lds, turn);
    const float along = s[0] * inv_cols, mean = s[1] * inv_cols;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) g[k][i] = (__builtin_fmaf(-along, h[k][i], g[k][i]) - mean) * rstd;
}

template <class T> __device__ __forceinline__ void store_grad8(T *p, uint32_t n, float (&v)[8], bool add)
{
    if (add) {
        float o[8];
        unpack8(load8(p, n), o);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += o[i];
    }
    store8(p, n, v);
}

template <class TX, class TF, int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES == 1 ? BACKWARD_TEAMS * 64 : WAVES * 64) void k_edge_backward(BackwardArgs a)
{
    constexpr uint32_t TEAMS = WAVES == 1 ? BACKWARD_TEAMS : 1;
    __shared__ float lds[2][2][WAVES];
    uint32_t turn = 0;
    const uint32_t team = uniform(threadIdx.x / (WAVES * 64));
    const EdgeLayer &l = a.l;
    uint32_t c[CHUNKS], n[CHUNKS];
    float wp[CHUNKS][8], bp[CHUNKS][8], wn[CHUNKS][8];
    float acc[ACCS][CHUNKS][8];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        c[k] = Team<WAVES, CHUNKS>::col(k);
        n[k] = live8(c[k], l.cols);
        if (l.post_weight) load8_f32(l.post_weight + c[k], n[k], wp[k]);
        if (l.post_bias) load8_f32(l.post_bias + c[k], n[k], bp[k]);
        if (l.pre_weight) load8_f32(l.pre_weight + c[k], n[k], wn[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!l.post_weight) wp[k][i] = 1.0f;
            if (!l.post_bias) bp[k][i] = 0.0f;
            if (!l.pre_weight) wn[k][i] = 1.0f;
#pragma unroll
            for (int q = 0; q < ACCS; ++q) acc[q][k][i] = 0.0f;
        }
    }
    // this team's rows: first, the distance to the next one, where they end; then the same of the next gate row
    const Cut &cut = a.cut;
    uint32_t gate_row, row, end, gate_end;
    const uint32_t step = cut.whole ? 1u : TEAMS;
    if (cut.whole) {
        gate_row = blockIdx.x * cut.whole + team;
        gate_end = min(cut.gates, (blockIdx.x + 1) * cut.whole);
        row = gate_row < gate_end ? gate_row * cut.rows_per_gate : a.rows;
        end = min(a.rows - row, cut.rows_per_gate) + row;
    } else {
        gate_row = blockIdx.x / cut.parts;
        gate_end = 0;
        const uint32_t first = gate_row * cut.rows_per_gate, part = (blockIdx.x - gate_row * cut.parts) * cut.run;
        // (parts behind the last row of a short last gate row are empty)
        const uint32_t of_gate = min(a.rows - first, cut.rows_per_gate);
        row = first + min(part + team, of_gate);
        end = first + min(part + cut.run, of_gate);
    }
    BackwardRow<TX, TF, CHUNKS> next;
    bool more = row < end;
    if (more) fetch<TX, TF, WAVES, CHUNKS>(next, a, row, c, n);
    while (more) {
        const BackwardRow<TX, TF, CHUNKS> now = next;
        const uint32_t this_row = row, this_gate = gate_row;
        row += step;
        bool gate_done = false;
        if (row >= end) {
            gate_done = cut.whole != 0;
            more = false;
            if (cut.whole) {
                gate_row += TEAMS;
                if (gate_row < gate_end) {
                    row = gate_row * cut.rows_per_gate;
                    end = min(a.rows - row, cut.rows_per_gate) + row;
                    more = true;
                }
            }
        }
        if (more) fetch<TX, TF, WAVES, CHUNKS>(next, a, row, c, n);

        // d: through the stream's norm
        float d[CHUNKS][8], h[CHUNKS][8];
        if (a.du) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                unpack8(now.u[k], d[k]);
                unpack_kept<TX>(now.x[k], a.pre_codes, l.pre, now.stats.z, now.stats.w, n[k], h[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    acc[ACC_PRE_WEIGHT][k][i] = __builtin_fmaf(d[k][i], h[k][i], acc[ACC_PRE_WEIGHT][k][i]);
                    acc[ACC_PRE_BIAS][k][i] += d[k][i];
                    d[k][i] *= wn[k][i];
                }
            }
            through_norm<WAVES, CHUNKS>(d, h, l.pre, now.stats.w, l.inv_cols, lds, turn);
        } else {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[k][i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            if (a.dx_out) {
                float o[8];
                unpack8(now.d[k], o);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[k][i] += o[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) d[k][i] = (uint32_t)i < n[k] ? d[k][i] : 0.0f;
            if (a.dx) {
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = l.skip * d[k][i];
                store8((TX *)a.dx + this_row * a.dx_stride + c[k], n[k], o);
            }
        }
        // m and k: through the gate and the branch's norm
        if (a.branch) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                unpack_kept<TF>(now.f[k], a.post_codes, l.post, now.stats.x, now.stats.y, n[k], h[k]);
                float g[8];
                if (a.gate) unpack_gate<TF>(now.g[k], a.gate_f32, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    d[k][i] *= l.branch;
                    acc[ACC_GATE][k][i] = __builtin_fmaf(d[k][i], __builtin_fmaf(h[k][i], wp[k][i], bp[k][i]), acc[ACC_GATE][k][i]);
                    if (a.gate) d[k][i] *= g[i];
                    acc[ACC_POST_WEIGHT][k][i] = __builtin_fmaf(d[k][i], h[k][i], acc[ACC_POST_WEIGHT][k][i]);
                    acc[ACC_POST_BIAS][k][i] += d[k][i];
                    d[k][i] *= wp[k][i];
                }
            }
            through_norm<WAVES, CHUNKS>(d, h, l.post, now.stats.y, l.inv_cols, lds, turn);
            if (a.df) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) store8((TF *)a.df + this_row * a.df_stride + c[k], n[k], d[k]);
            }
            if (gate_done) {
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) {
                    if (a.dgate) {
                        const uint64_t at = this_gate * a.dgate_stride + c[k];
                        if (a.gate_f32) store_grad8((float *)a.dgate + at, n[k], acc[ACC_GATE][k], a.accumulate);
                        else store_grad8((TF *)a.dgate + at, n[k], acc[ACC_GATE][k], false);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[ACC_GATE][k][i] = 0.0f;
                }
            }
        }
    }

    // what this workgroup adds up to: the teams' sums, then to its place among the partial sums
    __shared__ float sums[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? CHUNKS * 512 : 1];
#pragma unroll
    for (int q = 0; q < ACCS; ++q) {
        if (q < ACC_GATE ? !a.grad[q < ACC_GATE ? q : 0] : (!a.dgate || cut.whole)) continue;
        float *to = a.partial + ((uint64_t)q * cut.blocks + blockIdx.x) * l.cols;
        if constexpr (TEAMS > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[team][c[k] + i] = acc[q][k][i];
            __syncthreads();
            for (uint32_t j = threadIdx.x; j < l.cols; j += TEAMS * 64) {
                float s = sums[0][j];
#pragma unroll
                for (uint32_t t = 1; t < TEAMS; ++t) s += sums[t][j];
                to[j] = s;
            }
        } else {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) store8(to + c[k], n[k], acc[q][k]);
        }
    }
}

// Adds up the workgroups' partial sums, 64 columns and REDUCE_LINES lines at a time; blockIdx.y: one of the four parameter
// gradients, then the gate rows whose gradients are in parts.
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

// Wavefronts of a row's team (8 columns a lane, two rounds of them beyond 512).
static uint32_t waves_of(uint32_t cols)
{
    uint32_t w = 1;
    while (w * 1024 < cols) w *= 2;
    return w;
}

// Workgroups of the backward pass.
static Cut cut_of(uint32_t rows, uint32_t cols, uint32_t rows_per_gate)
{
    const uint32_t waves = waves_of(cols), teams = waves == 1 ? BACKWARD_TEAMS : 1u;
    const uint32_t most = waves == 1 ? 256u : waves == 2 ? 1024u : waves == 4 ? 512u : 256u;
    Cut t;
    t.rows_per_gate = rows_per_gate && rows_per_gate < rows ? rows_per_gate : rows;
    t.gates = (rows - 1) / t.rows_per_gate + 1;
    t.whole = t.parts = t.run = 0;
    if (t.gates >= most) {
        t.whole = (t.gates + most - 1) / most;
        if (teams > 1) t.whole = (t.whole + teams - 1) / teams * teams;
        t.blocks = (t.gates + t.whole - 1) / t.whole;
    } else {
        const uint32_t rounds = (t.rows_per_gate + teams - 1) / teams;      // of a team, if one workgroup took a gate row
        t.parts = most / t.gates < rounds ? most / t.gates : rounds;
        t.run = (rounds + t.parts - 1) / t.parts * teams;
        t.parts = (t.rows_per_gate + t.run - 1) / t.run;
        t.blocks = t.gates * t.parts;
    }
    return t;
}

template <class TX, class TF> static void launch_forward(const ForwardArgs &a, hipStream_t st)
{
    const uint32_t waves = waves_of(a.l.cols), teams = waves == 1 ? FORWARD_TEAMS : 1u;
    const uint32_t need = (a.rows + teams - 1) / teams, most = 4096u / (teams * waves);
    const dim3 grid(need < most ? need : most);
    if (a.l.cols <= 512) hipLaunchKernelGGL((k_edge_forward<TX, TF, 1, 1>), grid, dim3(FORWARD_TEAMS * 64), 0, st, a);
    else if (waves == 1) hipLaunchKernelGGL((k_edge_forward<TX, TF, 1, 2>), grid, dim3(FORWARD_TEAMS * 64), 0, st, a);
    else if (waves == 2) hipLaunchKernelGGL((k_edge_forward<TX, TF, 2, 2>), grid, dim3(128), 0, st, a);
    else if (waves == 4) hipLaunchKernelGGL((k_edge_forward<TX, TF, 4, 2>), grid, dim3(256), 0, st, a);
    else if (waves == 8) hipLaunchKernelGGL((k_edge_forward<TX, TF, 8, 2>), grid, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((k_edge_forward<TX, TF, 16, 2>), grid, dim3(1024), 0, st, a);
}

template <class TX, class TF> static void launch_backward(const BackwardArgs &a, hipStream_t st)
{
    const uint32_t waves = waves_of(a.l.cols);
    const dim3 grid(a.cut.blocks);
    if (a.l.cols <= 512) hipLaunchKernelGGL((k_edge_backward<TX, TF, 1, 1>), grid, dim3(BACKWARD_TEAMS * 64), 0, st, a);
    else if (waves == 1) hipLaunchKernelGGL((k_edge_backward<TX, TF, 1, 2>), grid, dim3(BACKWARD_TEAMS * 64), 0, st, a);
    else if (waves == 2) hipLaunchKernelGGL((k_edge_backward<TX, TF, 2, 2>), grid, dim3(128), 0, st, a);
    else if (waves == 4) hipLaunchKernelGGL((k_edge_backward<TX, TF, 4, 2>), grid, dim3(256), 0, st, a);
    else if (waves == 8) hipLaunchKernelGGL((k_edge_backward<TX, TF, 8, 2>), grid, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((k_edge_backward<TX, TF, 16, 2>), grid, dim3(1024), 0, st, a);
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
    if (e.cols > DGS_EDGE_MAX_COLS || !types_have(p.stream_type, p.type)) return DGS_ENOTSUP;
    ForwardArgs a;
    a.l = layer_of(e);
    a.x = p.x.data; a.f = p.f.data; a.gate = p.gate.data; a.x_out = p.x_out.data; a.u = p.u.data;
    a.post_codes = p.post_saved.codes; a.post_exps = p.post_saved.exps;
    a.pre_codes = p.pre_saved.codes; a.pre_exps = p.pre_saved.exps;
    a.stats = p.stats;
    a.x_stride = p.x.stride; a.f_stride = p.f.stride; a.gate_stride = p.gate.stride;
    a.x_out_stride = p.x_out.stride; a.u_stride = p.u.stride;
    a.post_codes_stride = p.post_saved.codes_stride; a.post_exps_stride = p.post_saved.exps_stride;
    a.pre_codes_stride = p.pre_saved.codes_stride; a.pre_exps_stride = p.pre_saved.exps_stride;
    a.rows = p.rows;
    a.rows_per_gate = p.gate.data ? p.rows_per_gate : 1u;
    a.gate_f32 = p.gate_type == DGS_F32;
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
    if (through_pre && e.pre == DGS_NORM_NONE) return DGS_EINVAL;
    if (!branch && (e.post != DGS_NORM_NONE || p.gate.data || p.df.data || p.post_weight_grad || p.post_bias_grad)) return DGS_EINVAL;
    if (p.dgate.data && !p.gate.data) return DGS_EINVAL;
    if (!aligned_to(p.post_weight_grad, 4) || !aligned_to(p.post_bias_grad, 4) || !aligned_to(p.pre_weight_grad, 4)
        || !aligned_to(p.pre_bias_grad, 4))
        return DGS_EINVAL;
    if (p.rows) {
        if (!present_ok(p.dx_out, cols, p.stream_type) || !present_ok(p.du, cols, p.type) || !present_ok(p.dx, cols, p.stream_type)
            || !present_ok(p.df, cols, p.type) || !gate_ok(p.gate, cols, p.gate_type, p.type, p.rows_per_gate)
            || !present_ok(p.dgate, cols, p.gate_type))
            return DGS_EINVAL;
        // one of the two per norm
        if (branch && (p.post_saved.codes ? p.f.data || !codes_ok(p.post_saved, cols) : !matrix_ok(p.f.data, p.f.stride, cols, p.type)))
            return DGS_EINVAL;
        if (through_pre
            && (p.pre_saved.codes ? p.x_out.data || !codes_ok(p.pre_saved, cols)
                                  : !matrix_ok(p.x_out.data, p.x_out.stride, cols, p.stream_type)))
            return DGS_EINVAL;
        if (!p.stats || !aligned_to(p.stats, 4)) return DGS_EINVAL;
    }
    if (e.cols > DGS_EDGE_MAX_COLS || !types_have(p.stream_type, p.type)) return DGS_ENOTSUP;
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
        a.dx_out_stride = p.dx_out.stride; a.du_stride = p.du.stride; a.gate_stride = p.gate.stride; a.f_stride = p.f.stride;
        a.x_out_stride = p.x_out.stride; a.dx_stride = p.dx.stride; a.df_stride = p.df.stride; a.dgate_stride = p.dgate.stride;
        a.post_codes_stride = p.post_saved.codes_stride; a.post_exps_stride = p.post_saved.exps_stride;
        a.pre_codes_stride = p.pre_saved.codes_stride; a.pre_exps_stride = p.pre_saved.exps_stride;
        a.rows = p.rows;
        a.gate_f32 = p.gate_type == DGS_F32;
        a.accumulate = p.accumulate != 0;
        a.branch = branch;
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
    const uint32_t in_parts = p.rows && p.dgate.data && !a.cut.whole ? a.cut.gates : 0u;
    if (grads || in_parts)
        hipLaunchKernelGGL(k_edge_reduce, dim3((e.cols + 63) / 64, 4 + in_parts), dim3(REDUCE_LINES * 64), 0, st,
                           (const float *)p.workspace, p.post_weight_grad, p.post_bias_grad, p.pre_weight_grad, p.pre_bias_grad,
                           p.dgate.data, p.dgate.stride, e.cols, p.rows ? a.cut.blocks : 0u, p.rows ? a.cut.parts : 0u,
                           (uint32_t)p.gate_type, (uint32_t)(p.accumulate != 0));
    return launched();
}
