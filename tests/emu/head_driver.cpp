// The output layer's and the orthogonalising kernels on the CPU, through the C ABI: every buffer an exact-size heap block (rows of
// a matrix apart by more than they are long, the last one ending where the block ends), every result against a plain
// computation in double.
#include <hip/hip_runtime.h>
#include "../../include/dgs_blocks.h"
#include <memory>
#include <random>
#include <string>

static std::mt19937 gen(11);
static double normal() { static std::normal_distribution<double> d; return d(gen); }

static double read_as(int type, const void *p, uint64_t i)
{
    if (type == DGS_F32) return ((const float *)p)[i];
    const uint16_t h = ((const uint16_t *)p)[i];
    if (type == DGS_BF16) return __uint_as_float((uint32_t)h << 16);
    _Float16 f;
    memcpy(&f, &h, 2);
    return (double)f;
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
static double half_step(int type) { return type == DGS_F32 ? ldexp(1.0, -24) : type == DGS_F16 ? ldexp(1.0, -11) : ldexp(1.0, -8); }

// A matrix; `shift` elements behind a 16-byte boundary.
struct Mat {
    int type;
    uint64_t rows, cols, stride;
    std::unique_ptr<char[]> store;
    char *p;
    Mat(int t, uint64_t r, uint64_t c, uint64_t pad, uint64_t shift, bool fill, double scale = 1.0) : type(t), rows(r), cols(c), stride(c + pad)
    {
        const uint64_t b = t == DGS_F32 ? 4 : 2, n = r ? (r - 1) * stride + c : 0;
        store.reset(new char[(n + shift) * b + (n + shift == 0)]);
        p = store.get() + shift * b;
        memset(p, 0x7F, n * b);
        if (fill)
            for (uint64_t i = 0; i < r; ++i)
                for (uint64_t j = 0; j < c; ++j) write_as(t, p, i * stride + j, scale * normal());
    }
    double at(uint64_t i, uint64_t j) const { return read_as(type, p, i * stride + j); }
    void set(uint64_t i, uint64_t j, double v) { write_as(type, p, i * stride + j, v); }
    dgs_matrix view() { return dgs_matrix{p, stride}; }
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
static void expect(int rc, const char *what)
{
    if (rc == DGS_OK) return;
    printf("%s: %s returned %d\n", name.c_str(), what, rc);
    exit(1);
}

static void head(int type, uint32_t rows, uint32_t cols, uint32_t vocab, uint32_t pad, uint32_t shift, bool bias, bool wide, bool add)
{
    name = "head " + std::to_string(type) + " " + std::to_string(rows) + "x" + std::to_string(cols) + "x" + std::to_string(vocab);
    Mat x(type, rows, cols, pad, shift, true, 1.0), w(type, vocab, cols, pad, 0, true, 1.0 / sqrt((double)cols));
    Mat b(DGS_F32, 1, vocab, 0, 0, true, 0.5), dloss(DGS_F32, 1, rows, 0, 0, true), dlse(DGS_F32, 1, rows, 0, 0, true, 0.1);
    Mat loss(DGS_F32, 1, rows, 0, 0, false), lse(DGS_F32, 1, rows, 0, 0, false);
    Mat dx(type, rows, cols, pad, shift, false), dw(DGS_F32, vocab, cols, pad, 1, true), db(DGS_F32, 1, vocab, 0, 0, true);
    std::unique_ptr<char[]> targets(new char[rows * (wide ? 8 : 4) + 1]);
    std::vector<long> target(rows);
    for (uint32_t t = 0; t < rows; ++t) {
        target[t] = t % 5 == 3 ? (t % 2 ? -100 : (long)vocab) : (long)(gen() % vocab);
        if (t == 0) target[t] = vocab - 1;
        if (wide) ((int64_t *)targets.get())[t] = target[t];
        else ((int32_t *)targets.get())[t] = (int32_t)target[t];
        if (t % 7 == 4) dloss.set(0, t, 0.0), dlse.set(0, t, 0.0);      // nothing arrives
        if (t % 11 == 9) dloss.set(0, t, 1e-9 * normal());
    }
    if (bias && vocab > 3) b.set(0, 2, -INFINITY);
    std::vector<double> dw0(vocab * cols), db0(vocab);
    for (uint32_t v = 0; v < vocab; ++v) {
        db0[v] = add ? db.at(0, v) : 0.0;
        for (uint32_t c = 0; c < cols; ++c) dw0[v * cols + c] = add ? dw.at(v, c) : 0.0;
    }
    dgs_head_args a = {};
    a.rows = rows; a.cols = cols; a.vocab = vocab;
    a.type = type; a.target_bytes = wide ? 8 : 4; a.accumulate = add;
    a.x = x.view(); a.weight = w.view();
    a.bias = bias ? (const float *)b.p : nullptr;
    a.targets = targets.get();
    a.loss = (float *)loss.p; a.lse = (float *)lse.p;
    auto with_workspace = [&](int back) {
        const uint64_t n = dgs_head_workspace(&a, back);
        std::unique_ptr<char[]> ws(new char[n + 256]);
        memset(ws.get(), 0xFF, n + 256);
        a.workspace = ws.get() + (-(uintptr_t)ws.get() & 15u);
        a.workspace_bytes = n;
        expect(back ? dgs_head_backward(&a, nullptr) : dgs_head_forward(&a, nullptr), back ? "backward" : "forward");
    };
    with_workspace(0);
    // logits' error: products of 22 bits a factor for fp32, sums of `cols` fp32 additions
    std::vector<double> z(rows * vocab), dz(rows * vocab);
    for (uint32_t t = 0; t < rows; ++t) {
        double top = -INFINITY, sum = 0.0, size = 0.0;
        for (uint32_t v = 0; v < vocab; ++v) {
            double s = bias ? b.at(0, v) : 0.0, m = std::isfinite(s) ? std::fabs(s) : 0.0;
            for (uint32_t c = 0; c < cols; ++c) s += x.at(t, c) * w.at(v, c), m += std::fabs(x.at(t, c) * w.at(v, c));
            z[t * vocab + v] = s;
            top = std::max(top, s);
            size = std::max(size, m);
        }
        for (uint32_t v = 0; v < vocab; ++v) sum += exp(z[t * vocab + v] - top);
        const double l = top + log(sum), tol = ldexp(size * (cols + 8), -24) + ldexp(std::fabs(l) + 40.0, -22);
        near(lse.at(0, t), l, tol, "lse", t);
        const bool counts = target[t] >= 0 && target[t] < (long)vocab;
        const double want = counts ? l - z[t * vocab + target[t]] : 0.0;
        if (std::isinf(want)) near(std::isinf(loss.at(0, t)), 1.0, 0.0, "infinite loss", t);
        else near(loss.at(0, t), want, counts ? 2 * tol : 0.0, "loss", t);
        const double up = counts ? dloss.at(0, t) : 0.0;
        for (uint32_t v = 0; v < vocab; ++v) dz[t * vocab + v] = (up + dlse.at(0, t)) * exp(z[t * vocab + v] - l) - ((long)v == target[t] ? up : 0.0);
    }
    a.dloss = (const float *)dloss.p;
    a.dlse = (const float *)dlse.p;
    a.dx = dx.view();
    a.dweight = (float *)dw.p;
    a.dweight_stride = dw.stride;
    a.dbias = (float *)db.p;
    with_workspace(1);
    const double rel = 1e-5;      // of dz, from the logits' own error (their size is below 10)
    for (uint32_t t = 0; t < rows; ++t)
        for (uint32_t c = 0; c < cols; ++c) {
            double s = 0.0, m = 0.0;
            for (uint32_t v = 0; v < vocab; ++v) s += dz[t * vocab + v] * w.at(v, c), m += std::fabs(dz[t * vocab + v] * w.at(v, c));
            near(dx.at(t, c), s, m * (rel + (type == DGS_F32 ? 0.0 : ldexp(1.0, -11))) + std::fabs(s) * 2 * half_step(type) + 1e-12 + (type == DGS_F16 ? ldexp(1.0, -24) : 0.0), "dx", t, c);
        }
    for (uint32_t v = 0; v < vocab; ++v) {
        double s = 0.0, m = 0.0;
        for (uint32_t t = 0; t < rows; ++t) s += dz[t * vocab + v], m += std::fabs(dz[t * vocab + v]);
        near(db.at(0, v), db0[v] + s, m * rel + std::fabs(db0[v]) * 1e-6, "dbias", v);
        for (uint32_t c = 0; c < cols; ++c) {
            s = m = 0.0;
            for (uint32_t t = 0; t < rows; ++t) s += dz[t * vocab + v] * x.at(t, c), m += std::fabs(dz[t * vocab + v] * x.at(t, c));
            near(dw.at(v, c), dw0[v * cols + c] + s, m * rel + std::fabs(dw0[v * cols + c]) * 1e-6 + 1e-12, "dweight", v, c);
        }
    }
}

static void ortho(int type, int out_type, uint32_t count, uint32_t rows, uint32_t cols, uint32_t pad, uint32_t steps, bool add)
{
    name = "ortho " + std::to_string(type) + "-" + std::to_string(out_type) + " " + std::to_string(count) + "x" + std::to_string(rows) + "x" + std::to_string(cols);
    const double A = 3.4445, B = -4.7750, C = 2.0315;
    std::vector<std::unique_ptr<Mat>> in, out, before;
    std::vector<dgs_matrix> vi, vo;
    for (uint32_t i = 0; i < count; ++i) {
        in.emplace_back(new Mat(type, rows, cols, pad + i, i, true, i == 1 ? 0.0 : 0.01));
        out.emplace_back(new Mat(out_type, rows, cols, pad, 0, true));
        before.emplace_back(new Mat(DGS_F32, rows, cols, 0, 0, false));
        for (uint32_t r = 0; r < rows; ++r)
            for (uint32_t c = 0; c < cols; ++c) before[i]->set(r, c, add ? out[i]->at(r, c) : 0.0);
        vi.push_back(in[i]->view());
        vo.push_back(out[i]->view());
    }
    dgs_orthogonalise_args a = {};
    a.count = count; a.rows = rows; a.cols = cols; a.steps = steps;
    a.type = type; a.out_type = out_type; a.accumulate = add;
    a.a = (float)A; a.b = (float)B; a.c = (float)C; a.eps = 1e-7f; a.scale = 0.5f;
    a.in = vi.data(); a.out = vo.data();
    const uint64_t n = dgs_orthogonalise_workspace(&a);
    std::unique_ptr<char[]> ws(new char[n + 256]);
    memset(ws.get(), 0xFF, n + 256);
    a.workspace = ws.get() + (-(uintptr_t)ws.get() & 15u);
    a.workspace_bytes = n;
    expect(dgs_orthogonalise(&a, nullptr), "orthogonalise");
    for (uint32_t i = 0; i < count; ++i) {
        const bool turned = rows > cols;
        const uint32_t m = turned ? cols : rows, k = turned ? rows : cols;
        std::vector<double> x(m * k), g(m * m), p(m * m), y(m * k);
        double norm = 0.0;
        for (uint32_t r = 0; r < rows; ++r)
            for (uint32_t c = 0; c < cols; ++c) {
                const double v = in[i]->at(r, c);
                norm += v * v;
                (turned ? x[c * k + r] : x[r * k + c]) = v;
            }
        for (double &v : x) v /= sqrt(norm) + 1e-7;
        for (uint32_t s = 0; s < steps; ++s) {
            for (uint32_t r = 0; r < m; ++r)
                for (uint32_t c = 0; c < m; ++c) {
                    double d = 0.0;
                    for (uint32_t j = 0; j < k; ++j) d += x[r * k + j] * x[c * k + j];
                    g[r * m + c] = d;
                }
            for (uint32_t r = 0; r < m; ++r)
                for (uint32_t c = 0; c < m; ++c) {
                    double d = 0.0;
                    for (uint32_t j = 0; j < m; ++j) d += g[r * m + j] * g[j * m + c];
                    p[r * m + c] = a.b * g[r * m + c] + a.c * d + (r == c ? a.a : 0.0);
                }
            for (uint32_t r = 0; r < m; ++r)
                for (uint32_t j = 0; j < k; ++j) {
                    double d = 0.0;
                    for (uint32_t c = 0; c < m; ++c) d += p[r * m + c] * x[c * k + j];
                    y[r * k + j] = d;
                }
            x = y;
        }
        double off = 0.0, size = 0.0;
        for (uint32_t r = 0; r < rows; ++r)
            for (uint32_t c = 0; c < cols; ++c) {
                const double want = before[i]->at(r, c) + 0.5 * (turned ? x[c * k + r] : x[r * k + c]), got = out[i]->at(r, c);
                if (!std::isfinite(got)) near(got, want, 0.0, "finite", r, c);
                off += (got - want) * (got - want);
                size += want * want;
            }
        // relative to the whole: rounding of the result, and of the products' operands, grown by as much as the small singular values
        near(sqrt(off), 0.0, sqrt(size) * (out_type == DGS_BF16 ? 6e-3 : out_type == DGS_F16 ? 5e-4 : 5e-5), "distance", i);
    }
}

int main(int, char **argv)
{
    const std::string what = argv[1];
    if (what == "head") {
        for (int type = 0; type < 3; ++type) {
            head(type, 1, 8, 5, 0, 0, false, true, false);
            head(type, 3, 1, 1, 0, 0, true, false, false);
            head(type, 37, 70, 133, 0, 0, true, true, true);
            head(type, 33, 64, 300, 3, 1, false, false, false);
            head(type, 140, 72, 129, 8, 8, true, false, true);
        }
        head(2, 32, 136, 260, 0, 0, false, true, false);
        // few rows, operands as they are: whole chunks and what is left of them, any alignment
        for (int type = 0; type < 3; ++type) {
            head(type, 5, 300, 140, 1, 1, true, true, true);
            head(type, 17, 129, 70, 3, 0, true, false, false);
            head(type, 32, 257, 45, 0, 1, false, true, false);
        }
        head(2, 0, 16, 9, 0, 0, true, true, false);
        head(1, 0, 16, 9, 0, 0, true, true, true);
    } else if (what == "large") {
        head(2, 270, 72, 300, 0, 0, true, true, false);
        head(1, 257, 64, 257, 8, 0, false, true, true);
        head(0, 30, 40, 520, 0, 0, true, true, false);
    } else if (what == "tiles") {
        ortho(0, 0, 2, 133, 40, 1, 2, false);
        ortho(2, 2, 1, 130, 140, 0, 1, true);
    } else {
        for (int out = 0; out < 3; ++out) {
            ortho(0, out, 1, 1, 1, 0, 5, false);
            ortho(out, out, 3, 5, 70, 0, 5, true);
            ortho(2 - out, out, 2, 133, 40, 1, 5, false);
            ortho(0, out, 1, 130, 140, 0, 2, false);
            // whole matrices to a workgroup
            ortho(out, out, 2, 100, 77, 3, 3, false);
            ortho(2 - out, out, 1, 128, 128, 0, 1, true);
            ortho(0, out, 2, 64, 33, 1, 4, false);
            ortho(out, out, 1, 17, 129, 0, 2, false);
        }
    }
    printf("%llu values as expected\n", (unsigned long long)checks);
    return 0;
}
