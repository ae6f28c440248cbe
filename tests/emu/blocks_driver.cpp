// The training-block kernels on the CPU, through the C ABI: every buffer an exact-size heap block (rows of a matrix apart by
// more than they are long, the last one ending where the block ends), every result against a plain computation in double.
#include <hip/hip_runtime.h>
#include "../../include/dgs_blocks.h"
#include <memory>
#include <random>

static std::mt19937 gen(7);
static double normal() { static std::normal_distribution<double> d; return d(gen); }

static float half_to_float(uint16_t h)
{
    _Float16 f;
    memcpy(&f, &h, 2);
    return (float)f;
}
static double read_as(int type, const void *p, uint64_t i)
{
    if (type == DGS_F32) return ((const float *)p)[i];
    const uint16_t h = ((const uint16_t *)p)[i];
    return type == DGS_F16 ? half_to_float(h) : __uint_as_float((uint32_t)h << 16);
}
static void write_as(int type, void *p, uint64_t i, double v)
{
    if (type == DGS_F32) {
        ((float *)p)[i] = (float)v;
    } else if (type == DGS_F16) {
        const _Float16 f = (_Float16)(float)v;
        memcpy((uint16_t *)p + i, &f, 2);
    } else {
        ((uint16_t *)p)[i] = (uint16_t)(__float_as_uint((float)v) >> 16);
    }
}

struct Mat {
    int type;
    uint64_t rows, cols, stride;
    std::unique_ptr<char[]> store;
    char *p;
    Mat(int t, uint64_t r, uint64_t c, uint64_t pad, bool fill, double scale = 1.0) : type(t), rows(r), cols(c), stride(c + pad)
    {
        const uint64_t b = t == DGS_F32 ? 4 : 2, n = r ? (r - 1) * stride + c : 0;
        store.reset(new char[n * b + 1]);
        p = store.get();
        memset(p, 0x7F, n * b);
        if (fill)
            for (uint64_t i = 0; i < r; ++i)
                for (uint64_t j = 0; j < c; ++j) write_as(t, p, i * stride + j, scale * normal());
    }
    double at(uint64_t i, uint64_t j) const { return read_as(type, p, i * stride + j); }
    dgs_matrix view() { return dgs_matrix{p, stride}; }
};

struct Codes {
    uint64_t rows, cols, runs;
    std::unique_ptr<int8_t[]> q;
    std::unique_ptr<uint8_t[]> e;
    uint64_t qs, es;
    Codes(uint64_t r, uint64_t c, uint64_t pad) : rows(r), cols(c), runs((c + 31) / 32), qs(c + pad), es((c + 31) / 32 + pad)
    {
        q.reset(new int8_t[r ? (r - 1) * qs + c : 1]);
        e.reset(new uint8_t[r ? (r - 1) * es + runs : 1]);
    }
    dgs_codes view() { return dgs_codes{q.get(), qs, e.get(), es}; }
    double at(uint64_t i, uint64_t j) const
    {
        const int b = e[i * es + j / 32];
        return b == 255 ? NAN : ldexp((double)q[i * qs + j], b - 127);
    }
    double step(uint64_t i, uint64_t j) const { return ldexp(1.0, (int)e[i * es + j / 32] - 127); }
};

static std::string name;
static uint64_t checks = 0;
static void near(double got, double want, double tol, const char *what, uint64_t i = 0, uint64_t j = 0)
{
    ++checks;
    if (std::isnan(want) ? std::isnan(got) : std::fabs(got - want) <= tol) return;
    printf("%s: %s (%llu, %llu): %.9g, expected %.9g within %.3g\n", name.c_str(), what, (unsigned long long)i, (unsigned long long)j, got,
           want, tol);
    exit(1);
}
static double eps_of(int type) { return type == DGS_F32 ? 6e-8 : type == DGS_F16 ? 4.9e-4 : 3.91e-3; }

struct Vec {
    std::unique_ptr<float[]> v;
    Vec(uint64_t n, double mean, double dev) : v(new float[n])
    {
        for (uint64_t i = 0; i < n; ++i) v[i] = (float)(mean + dev * normal());
    }
};

typedef std::vector<std::vector<double>> Grid;
static Grid grid(uint64_t r, uint64_t c) { return Grid(r, std::vector<double>(c, 0.0)); }

static void stats_of(const std::vector<double> &v, int kind, double eps, double &mean, double &rstd)
{
    mean = rstd = 0.0;
    if (kind == DGS_NORM_NONE) return;
    if (kind == DGS_NORM_LAYER) {
        for (double x : v) mean += x;
        mean /= (double)v.size();
    }
    double s = 0.0;
    for (double x : v) s += (x - mean) * (x - mean);
    rstd = 1.0 / std::sqrt(s / (double)v.size() + eps);
}

static void edge(uint32_t rows, uint32_t cols, int stream, int type, int post, int pre, bool bias, uint32_t rpg, bool gate32, bool coded,
                 uint64_t pad, bool branch = true)
{
    char buf[200];
    snprintf(buf, sizeof(buf), "edge %ux%u stream %d type %d post %d pre %d bias %d rpg %u gate32 %d coded %d pad %d branch %d", rows, cols,
             stream, type, post, pre, bias, rpg, gate32, coded, (int)pad, branch);
    name = buf;
    Mat x(stream, rows, cols, pad, true, 2.0), f(type, rows, cols, pad, true), xo(stream, rows, cols, pad, false), u(type, rows, cols, pad, false);
    const int gt = gate32 ? (int)DGS_F32 : type;
    const uint32_t gates = rpg ? (rows + rpg - 1) / rpg : 0;
    Mat g(gt, gates, cols, pad, true), dg(gt, gates, cols, pad, false);
    Vec wp(cols, 1, 0.2), bp(cols, 0, 0.1), wn(cols, 1, 0.2), bn(cols, 0, 0.1);
    Codes cp(rows, cols, pad), cn(rows, cols, pad);
    std::unique_ptr<float[]> stats(new float[4 * rows]);
    dgs_edge e = {};
    e.cols = cols; e.post = post; e.pre = pre; e.post_eps = e.pre_eps = 1e-5f; e.skip = 1.25f; e.branch = 0.75f;
    if (post) { e.post_weight = wp.v.get(); if (bias) e.post_bias = bp.v.get(); }
    if (pre) { e.pre_weight = wn.v.get(); if (bias) e.pre_bias = bn.v.get(); }
    dgs_edge_forward_args a = {};
    a.rows = rows; a.rows_per_gate = rpg; a.stream_type = stream; a.type = type; a.gate_type = gt;
    a.x = x.view();
    if (branch) { a.f = f.view(); a.x_out = xo.view(); if (rpg) a.gate = g.view(); }
    if (pre) a.u = u.view();
    if (coded) { if (branch) a.post_saved = cp.view(); if (pre) a.pre_saved = cn.view(); }
    a.stats = stats.get();
    near(dgs_edge_forward(&e, &a, nullptr), 0, 0, "return value");
    Grid fh = grid(rows, cols), xh = grid(rows, cols);
    std::vector<double> fm(rows), fr(rows), xm(rows), xr(rows);
    auto gate = [&](uint32_t i, uint32_t j) { return rpg && branch ? g.at(i / rpg, j) : 1.0; };
    auto wpost = [&](uint32_t j) { return post ? (double)wp.v[j] : 1.0; };
    auto bpost = [&](uint32_t j) { return post && bias ? (double)bp.v[j] : 0.0; };
    for (uint32_t i = 0; i < rows; ++i) {
        std::vector<double> v(cols);
        if (branch) {
            for (uint32_t j = 0; j < cols; ++j) v[j] = f.at(i, j);
            stats_of(v, post, 1e-5, fm[i], fr[i]);
            for (uint32_t j = 0; j < cols; ++j) fh[i][j] = post ? (v[j] - fm[i]) * fr[i] : v[j];
        }
        for (uint32_t j = 0; j < cols; ++j) {
            v[j] = x.at(i, j);
            if (branch) {
                v[j] = 1.25 * v[j] + 0.75 * gate(i, j) * (fh[i][j] * wpost(j) + bpost(j));
                near(xo.at(i, j), v[j], 2e-5 + std::fabs(v[j]) * eps_of(stream), "x_out", i, j);
            }
        }
        stats_of(v, pre, 1e-5, xm[i], xr[i]);
        near(stats[4 * i], fm[i], 1e-5, "post mean", i);
        near(stats[4 * i + 1], fr[i], 1e-5 * (1 + fr[i]), "post rstd", i);
        near(stats[4 * i + 2], xm[i], 1e-5, "pre mean", i);
        near(stats[4 * i + 3], xr[i], 1e-5 * (1 + xr[i]), "pre rstd", i);
        for (uint32_t j = 0; j < cols; ++j) {
            xh[i][j] = pre ? (v[j] - xm[i]) * xr[i] : 0.0;
            if (pre) {
                const double want = xh[i][j] * wn.v[j] + (bias ? bn.v[j] : 0.0);
                near(u.at(i, j), want, 2e-5 + std::fabs(want) * eps_of(type), "u", i, j);
            }
            if (coded) {
                if (branch) near(cp.at(i, j), fh[i][j], 0.51 * cp.step(i, j) + 1e-5, "post codes", i, j);
                if (pre) near(cn.at(i, j), xh[i][j], 0.51 * cn.step(i, j) + 1e-5, "pre codes", i, j);
            }
        }
    }
    // backward, with what the forward pass saved
    for (uint32_t i = 0; i < rows; ++i)
        for (uint32_t j = 0; j < cols; ++j) {
            if (branch) fh[i][j] = coded ? cp.at(i, j) : post ? (f.at(i, j) - stats[4 * i]) * stats[4 * i + 1] : f.at(i, j);
            if (pre) xh[i][j] = coded ? cn.at(i, j) : ((branch ? xo : x).at(i, j) - stats[4 * i + 2]) * stats[4 * i + 3];
        }
    Mat dxo(stream, rows, cols, pad, true), du(type, rows, cols, pad, true), dx(stream, rows, cols, pad, false), df(type, rows, cols, pad, false);
    Vec gw(cols, 0, 1), gb(cols, 0, 1), hw(cols, 0, 1), hb(cols, 0, 1);
    std::vector<float> gw0(gw.v.get(), gw.v.get() + cols), gb0(gb.v.get(), gb.v.get() + cols), hw0(hw.v.get(), hw.v.get() + cols),
        hb0(hb.v.get(), hb.v.get() + cols);
    const bool add = (rows & 1) != 0;
    if (gate32)
        for (uint32_t i = 0; i < gates; ++i)
            for (uint32_t j = 0; j < cols; ++j) write_as(DGS_F32, dg.p, i * dg.stride + j, 0.5);
    const size_t ws = dgs_edge_backward_workspace(rows, cols, rpg && branch ? rpg : 0);
    std::unique_ptr<char, void (*)(void *)> work((char *)aligned_alloc(16, (ws + 15) / 16 * 16), [](void *q) { free(q); });
    dgs_edge_backward_args b = {};
    b.rows = rows; b.rows_per_gate = rpg; b.stream_type = stream; b.type = type; b.gate_type = gt; b.accumulate = add;
    b.dx_out = dxo.view();
    if (pre) { b.du = du.view(); b.pre_weight_grad = hw.v.get(); if (bias) b.pre_bias_grad = hb.v.get(); }
    if (branch) {
        b.df = df.view();
        if (rpg) { b.gate = g.view(); b.dgate = dg.view(); }
        if (post) { b.post_weight_grad = gw.v.get(); if (bias) b.post_bias_grad = gb.v.get(); }
        if (coded) b.post_saved = cp.view(); else b.f = f.view();
    }
    if (pre) { if (coded) b.pre_saved = cn.view(); else b.x_out = (branch ? xo : x).view(); }
    b.stats = stats.get();
    b.dx = dx.view();
    b.workspace = work.get();
    b.workspace_bytes = ws;
    near(dgs_edge_backward(&e, &b, nullptr), 0, 0, "return value");
    std::vector<double> tw(cols), tb(cols), sw(cols), sb(cols);
    Grid tg = grid(gates, cols);
    auto through = [&](std::vector<double> &k, const std::vector<double> &h, int kind, double rstd) {
        if (!kind) return;
        double s = 0, m = 0;
        for (uint32_t j = 0; j < cols; ++j) { s += k[j] * h[j]; m += k[j]; }
        s /= cols;
        m = kind == DGS_NORM_LAYER ? m / cols : 0.0;
        for (uint32_t j = 0; j < cols; ++j) k[j] = rstd * (k[j] - m - h[j] * s);
    };
    for (uint32_t i = 0; i < rows; ++i) {
        std::vector<double> d(cols);
        if (pre) {
            for (uint32_t j = 0; j < cols; ++j) {
                sw[j] += du.at(i, j) * xh[i][j];
                sb[j] += du.at(i, j);
                d[j] = du.at(i, j) * wn.v[j];
            }
            through(d, xh[i], pre, stats[4 * i + 3]);
        }
        for (uint32_t j = 0; j < cols; ++j) {
            d[j] += dxo.at(i, j);
            near(dx.at(i, j), 1.25 * d[j], 1e-4 + std::fabs(d[j]) * 1.25 * eps_of(stream), "dx", i, j);
        }
        if (!branch) continue;
        for (uint32_t j = 0; j < cols; ++j) {
            if (rpg) tg[i / rpg][j] += 0.75 * d[j] * (fh[i][j] * wpost(j) + bpost(j));
            d[j] *= 0.75 * gate(i, j);
            tw[j] += d[j] * fh[i][j];
            tb[j] += d[j];
            d[j] *= wpost(j);
        }
        through(d, fh[i], post, stats[4 * i + 1]);
        for (uint32_t j = 0; j < cols; ++j) near(df.at(i, j), d[j], 1e-4 + std::fabs(d[j]) * eps_of(type), "df", i, j);
    }
    const double tol = 1e-4 * std::sqrt((double)rows) + 1e-4;
    for (uint32_t j = 0; j < cols; ++j) {
        if (branch && post) near(gw.v[j], tw[j] + (add ? gw0[j] : 0.0), tol, "post weight", j);
        if (branch && post && bias) near(gb.v[j], tb[j] + (add ? gb0[j] : 0.0), tol, "post bias", j);
        if (pre) near(hw.v[j], sw[j] + (add ? hw0[j] : 0.0), tol, "pre weight", j);
        if (pre && bias) near(hb.v[j], sb[j] + (add ? hb0[j] : 0.0), tol, "pre bias", j);
        if (branch)
            for (uint32_t i = 0; i < gates; ++i)
                near(dg.at(i, j), tg[i][j] + (add && gate32 ? 0.5 : 0.0), tol + std::fabs(tg[i][j]) * eps_of(gt), "dgate", i, j);
    }
}

static void checkpoint(uint32_t rows, uint32_t cols, int type, uint64_t pad, double scale, bool special)
{
    char buf[160];
    snprintf(buf, sizeof(buf), "checkpoint %ux%u type %d pad %d scale %g special %d", rows, cols, type, (int)pad, scale, special);
    name = buf;
    Mat x(type, rows, cols, pad, true, scale), out(DGS_F32, rows, cols, pad, false), back(type, rows, cols, pad, false);
    if (special) {
        const float inf = INFINITY;
        write_as(type, x.p, 0, NAN);
        if (cols > 40) write_as(type, x.p, 40, -inf);
        if (rows > 1)
            for (uint32_t j = 0; j < cols; ++j) write_as(type, x.p, x.stride + j, j % 2 ? -0.0 : 0.0);
    }
    Codes c(rows, cols, pad);
    const dgs_codes v = c.view();
    near(dgs_checkpoint_encode(rows, cols, type, x.p, x.stride, &v, nullptr), 0, 0, "return value");
    near(dgs_checkpoint_decode(rows, cols, &v, nullptr, nullptr, DGS_F32, out.p, out.stride, nullptr), 0, 0, "return value");
    Vec s(cols, 1, 0.2), b(cols, 0, 0.1);
    near(dgs_checkpoint_decode(rows, cols, &v, s.v.get(), b.v.get(), type, back.p, back.stride, nullptr), 0, 0, "return value");
    for (uint32_t i = 0; i < rows; ++i)
        for (uint32_t j0 = 0; j0 < cols; j0 += 32) {
            double top = 0;
            bool bad = false;
            const uint32_t j1 = std::min(cols, j0 + 32);
            for (uint32_t j = j0; j < j1; ++j) {
                bad |= !std::isfinite(x.at(i, j));
                top = std::max(top, std::fabs(x.at(i, j)));
            }
            int e = -126;
            while (!bad && e < 121 && top >= ldexp(127.5, e)) ++e;
            near(c.e[i * c.es + j0 / 32], bad ? 255 : e + 127, 0, "exponent byte", i, j0);
            for (uint32_t j = j0; j < j1; ++j) {
                const double q = bad ? 0 : std::max(-127.0, std::min(127.0, std::nearbyint(ldexp(x.at(i, j), -e))));
                near(c.q[i * c.qs + j], q, 0, "code", i, j);
                near(out.at(i, j), bad ? NAN : ldexp(q, e), 0, "value", i, j);
                const double w = bad ? NAN : ldexp(q, e) * s.v[j] + b.v[j];
                near(back.at(i, j), w, 1e-6 * scale + 1e-6 + std::fabs(w) * eps_of(type), "scaled value", i, j);
            }
        }
}

static void weight(uint32_t rows, uint32_t outs, uint32_t cols, int type, bool scaled, bool shifted, bool with_db, uint64_t pad, bool add)
{
    char buf[160];
    snprintf(buf, sizeof(buf), "weight %ux%ux%u type %d scale %d shift %d db %d pad %d add %d", rows, outs, cols, type, scaled, shifted, with_db,
             (int)pad, add);
    name = buf;
    Mat dy(type, rows, outs, pad, true), dw(DGS_F32, outs, cols, pad, true), x(DGS_F32, rows, cols, 0, true);
    Codes c(rows, cols, pad);
    const dgs_codes v = c.view();
    near(dgs_checkpoint_encode(rows, cols, DGS_F32, x.p, x.stride, &v, nullptr), 0, 0, "return value");
    Vec s(cols, 1, 0.2), b(cols, 0, 0.5), db(outs, 0, 1);
    Grid want = grid(outs, cols);
    std::vector<double> want_db(outs);
    for (uint32_t o = 0; o < outs; ++o) {
        want_db[o] = add ? db.v[o] : 0.0;
        for (uint32_t j = 0; j < cols; ++j) want[o][j] = add ? dw.at(o, j) : 0.0;
    }
    for (uint32_t i = 0; i < rows; ++i)
        for (uint32_t o = 0; o < outs; ++o) {
            const double d = dy.at(i, o);
            want_db[o] += d;
            for (uint32_t j = 0; j < cols; ++j) want[o][j] += d * (c.at(i, j) * (scaled ? s.v[j] : 1.0) + (shifted ? b.v[j] : 0.0));
        }
    const size_t ws = dgs_checkpoint_weight_grad_workspace(rows, outs, cols, type);
    std::unique_ptr<char, void (*)(void *)> work((char *)aligned_alloc(16, (ws + 15) / 16 * 16), [](void *q) { free(q); });
    dgs_weight_grad_args a = {};
    a.rows = rows; a.outs = outs; a.cols = cols; a.type = type; a.accumulate = add;
    a.dy = dy.view();
    a.saved = v;
    a.scale = scaled ? s.v.get() : nullptr;
    a.shift = shifted ? b.v.get() : nullptr;
    a.dw = (float *)dw.p;
    a.dw_stride = dw.stride;
    a.db = with_db ? db.v.get() : nullptr;
    a.workspace = work.get();
    a.workspace_bytes = ws;
    near(dgs_checkpoint_weight_grad(&a, nullptr), 0, 0, "return value");
    const double tol = 2e-6 * (std::sqrt((double)rows) + 1) * 4;
    for (uint32_t o = 0; o < outs; ++o) {
        for (uint32_t j = 0; j < cols; ++j) near(dw.at(o, j), want[o][j], tol, "dw", o, j);
        if (with_db) near(db.v[o], want_db[o], tol, "db", o);
    }
}

static const int F = DGS_F32, H = DGS_F16, B = DGS_BF16, R = DGS_NORM_RMS, L = DGS_NORM_LAYER;

static void checkpoints()
{
    for (int type : {F, H, B}) {
        checkpoint(1, 1, type, 0, 1.0, false);
        checkpoint(3, 31, type, 0, 1.0, true);
        checkpoint(2, 100, type, 5, 1e-3, true);
        checkpoint(5, 264, type, 1, 100.0, false);
        checkpoint(9, 1000, type, 0, 1.0, true);
    }
    checkpoint(3, 65, F, 0, 3e38, false);
    checkpoint(3, 65, B, 2, 1e-38, true);
}

// One wavefront a row, in one and two rounds; several; odd sizes, rows beyond one workgroup's share, short last gate rows, one
// workgroup alone, gate rows shared by teams and one to a team, wavefronts without a column.
static void edges()
{
    edge(1, 1, F, F, R, L, true, 0, false, true, 0);
    edge(5, 7, F, B, L, R, true, 2, false, true, 3);
    edge(67, 96, B, B, R, R, false, 0, false, true, 0);
    edge(8200, 8, F, B, L, R, true, 32, false, true, 0);
    edge(3, 96, H, H, R, L, true, 3, false, true, 1);
    edge(2, 700, B, B, R, L, true, 2, true, true, 1);
    edge(1, 8200, F, F, L, L, true, 1, true, true, 0);
    edge(2, 5000, B, B, L, L, true, 2, false, true, 0);
    edge(41, 333, H, H, L, L, true, 1, false, false, 1);
    edge(300, 40, F, H, L, L, true, 300, true, true, 8);
    edge(310, 33, B, B, R, L, true, 1, false, true, 0);
    edge(531, 24, F, F, L, R, true, 2, true, false, 0);
    edge(90, 768, F, B, L, L, true, 37, false, true, 0);
    edge(5, 1030, B, B, R, L, true, 0, false, true, 0);
    edge(4, 4300, F, B, L, R, true, 2, false, true, 0);
    edge(13, 1001, F, F, DGS_NORM_NONE, L, true, 4, true, true, 3);
    edge(9, 1500, B, B, R, R, false, 3, false, true, 0);
    edge(7, 2056, F, B, L, L, true, 0, false, false, 0);
    edge(6, 4100, H, H, R, L, true, 1, false, true, 5);
    edge(3, 8200, F, B, L, R, false, 3, true, true, 0);
    edge(8, 520, F, B, R, DGS_NORM_NONE, true, 8, true, true, 0);
    edge(8, 520, B, B, DGS_NORM_NONE, R, false, 0, false, true, 0);
    edge(11, 300, F, B, DGS_NORM_NONE, L, true, 0, false, true, 2, false);
    edge(11, 300, H, H, DGS_NORM_NONE, R, true, 0, false, false, 2, false);
}

// Rows too few for a step, tiles whole and cut, the bias terms in the launch and behind it, several splits of the rows.
static void weights()
{
    for (int type : {F, H, B}) {
        weight(1, 1, 1, type, false, false, true, 0, false);
        weight(33, 130, 70, type, true, true, true, 3, true);
        weight(300, 64, 136, type, true, false, true, 0, false);
        weight(700, 40, 33, type, false, true, false, 1, true);
    }
    weight(0, 5, 7, B, true, true, true, 0, false);
    weight(40, 140, 150, H, true, true, true, 1, false);
    weight(70, 300, 136, B, true, true, true, 0, true);
}

// The same for the large tiles (of a build in which they are taken at any size).
static void tiles()
{
    for (int type : {F, H, B}) {
        weight(64, 256, 256, type, true, true, true, 0, false);
        weight(300, 257, 150, type, true, true, true, 1, true);
        weight(330, 40, 264, type, true, false, true, 0, false);
    }
}

int main(int argc, char **argv)
{
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "edges") edges();
    else if (what == "weights") { checkpoints(); weights(); }
    else if (what == "tiles") tiles();
    else return 2;
    printf("%llu values as expected\n", (unsigned long long)checks);
    return 0;
}
