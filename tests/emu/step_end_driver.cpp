// Where numbers are hard for the orthogonalising kernels and the output layer's, on the CPU, through the C ABI: coefficients that take
// little or nothing off small singular values, against the same steps in double; entries of the vocabulary that are improbable, and
// fp32 weights of very unlike size, against the definition.
#include <hip/hip_runtime.h>
#include "../../include/dgs_blocks.h"
#include <functional>
#include <memory>
#include <random>
#include <string>

static std::mt19937 gen(17);
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
static double half_step(int type) { return type == DGS_F32 ? ldexp(1.0, -24) : type == DGS_F16 ? ldexp(1.0, -11) : ldexp(1.0, -8); }

static std::string name;
static uint64_t checks = 0;
static void near(double got, double want, double tol, const char *what, uint64_t i = 0, uint64_t j = 0)
{
    ++checks;
    if (std::fabs(got - want) <= tol) return;
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
// A call with a workspace of the size that it asks for, full of NaN.
static void with_workspace(uint64_t bytes, std::function<int(void *, uint64_t)> call, const char *what)
{
    std::unique_ptr<char[]> ws(new char[bytes + 16]);
    memset(ws.get(), 0xFF, bytes + 16);
    expect(call(ws.get() + (-(uintptr_t)ws.get() & 15u), bytes), what);
}

// An fp32 matrix of the given Frobenius norm.  A step rounds X by 2^-21 (bfloat16 results: 2^-10) for the operands, by 2^-24 sqrt(n) for a sum of n
// products (three pairs of parts; additions round to either side), and by 2^-37 of 1 since X's smallest values have fewer bits.  The
// result may be off by `grown` times the first two, relative to the whole, the steps' number times the last, and half a step of its type.
static void ortho(int out_type, uint32_t rows, uint32_t cols, float a, float b, float c, uint32_t steps, double norm, float eps, double grown)
{
    name = "ortho to " + std::to_string(out_type) + " " + std::to_string(rows) + "x" + std::to_string(cols) + " (" + std::to_string(a) + ", "
         + std::to_string(b) + ", " + std::to_string(c) + ")";
    std::vector<float> g(rows * cols);
    std::unique_ptr<char[]> out(new char[g.size() * (out_type == DGS_F32 ? 4 : 2)]);
    double sum = 0.0;
    for (float &v : g) v = (float)normal(), sum += (double)v * v;
    for (float &v : g) v = (float)(v * norm / sqrt(sum));
    dgs_matrix in = {g.data(), cols}, to = {out.get(), cols};
    dgs_orthogonalise_args p = {};
    p.count = 1; p.rows = rows; p.cols = cols; p.steps = steps;
    p.type = DGS_F32; p.out_type = out_type;
    p.a = a; p.b = b; p.c = c; p.eps = eps; p.scale = 1.0f;
    p.in = &in; p.out = &to;
    with_workspace(dgs_orthogonalise_workspace(&p), [&](void *ws, uint64_t n) { p.workspace = ws; p.workspace_bytes = n; return dgs_orthogonalise(&p, nullptr); }, "orthogonalise");
    const bool turned = rows > cols;
    const uint32_t m = turned ? cols : rows, k = turned ? rows : cols;
    std::vector<double> x(m * k), q(m * m), w(m * m), y(m * k);
    sum = 0.0;
    for (float v : g) sum += (double)v * v;
    for (uint32_t r = 0; r < rows; ++r)
        for (uint32_t j = 0; j < cols; ++j) (turned ? x[j * k + r] : x[r * k + j]) = g[r * cols + j] / (sqrt(sum) + (double)eps);
    for (uint32_t s = 0; s < steps; ++s) {
        for (uint32_t r = 0; r < m; ++r)
            for (uint32_t j = 0; j < m; ++j) {
                double d = 0.0;
                for (uint32_t i = 0; i < k; ++i) d += x[r * k + i] * x[j * k + i];
                q[r * m + j] = d;
            }
        for (uint32_t r = 0; r < m; ++r)
            for (uint32_t j = 0; j < m; ++j) {
                double d = 0.0;
                for (uint32_t i = 0; i < m; ++i) d += q[r * m + i] * q[i * m + j];
                w[r * m + j] = b * q[r * m + j] + c * d + (r == j ? a : 0.0);
            }
        for (uint32_t r = 0; r < m; ++r)
            for (uint32_t j = 0; j < k; ++j) {
                double d = 0.0;
                for (uint32_t i = 0; i < m; ++i) d += w[r * m + i] * x[i * k + j];
                y[r * k + j] = d;
            }
        x = y;
    }
    double far = 0.0, size = 0.0;
    for (uint32_t r = 0; r < rows; ++r)
        for (uint32_t j = 0; j < cols; ++j) {
            const double want = turned ? x[j * k + r] : x[r * k + j], got = read_as(out_type, out.get(), r * cols + j);
            if (!std::isfinite(got)) near(got, want, 0.0, "finite", r, j);
            const double d = std::max(0.0, std::fabs(got - want) - half_step(out_type) * std::fabs(want) - (out_type == DGS_F16 ? ldexp(1.0, -25) : 0.0));
            far += d * d;
            size += want * want;
        }
    near(sqrt(far), 0.0, sqrt(size) * grown * (ldexp(1.0, out_type == DGS_BF16 ? -10 : -21) + ldexp(sqrt(3.0 * k), -24)) + steps * ldexp(sqrt((double)(m * k)), -37), "distance");
}

// Singular values near 0 shrink or stay where others do not: up to 128 x 128 and beyond, rows or columns the smaller side.  What a step
// leaves grows as the map's slopes say, relative to X where X shrinks: by 2 a step at the fixed point 1 of (0.5, 0.5, 0); by 2 in all on the way to 0 of (0.75, 0.5, -0.25) from
// singular values of 0.42 and less (1 + 1.33 s^2 a step, with s^2 falling by a third each); (1, 0.9, -0.9) takes what 145 steps to 1 leave off
// again (slope -0.8 there); not at all far below 1.
static void coefficients()
{
    for (int out = 0; out < 3; ++out) {
        ortho(out, 1, 1, 0.5f, 0.5f, 0.0f, 7, 1.0, 1e-7f, 127);
        ortho(out, 1, 200, 0.5f, 0.5f, 0.0f, 10, 1.0, 1e-7f, 1023);
        ortho(out, 20, 30, 0.75f, 0.5f, -0.25f, 40, 1.0, 1e-7f, 80);
        ortho(out, 140, 9, 0.75f, 0.5f, -0.25f, 40, 1.0, 1e-7f, 80);
        // an update below eps whose X, at first a sixteenth, goes to 1 by way of b and c alone
        ortho(out, 1, 40, 1.0f, 0.9f, -0.9f, 180, 0.0661, 1.0f, 180);
        if (out == DGS_F32) ortho(out, 130, 1, 1.0f, 0.9f, -0.9f, 180, 0.0661, 1.0f, 180);
        // ... and ones far below it, which `a` alone moves
        ortho(out, 9, 20, 3.4445f, -4.7750f, 2.0315f, 5, 1e-9, 1.0f, 5);
        ortho(out, 9, 140, 3.4445f, -4.7750f, 2.0315f, 5, 1e-9, 1.0f, 5);
        ortho(out, 9, 20, 0.25f, 0.5f, 0.25f, 5, 1e-5, 1.0f, 5);
        ortho(out, 9, 140, 0.25f, 0.5f, 0.25f, 5, 1e-5, 1.0f, 5);
    }
}

// A matrix in memory, and its values as they are held.
struct Mat {
    int type;
    std::unique_ptr<char[]> store;
    std::vector<double> v;
    Mat(int t, uint64_t n, std::function<double(uint64_t)> value) : type(t), store(new char[n * (t == DGS_F32 ? 4 : 2) + 1]), v(n)
    {
        for (uint64_t i = 0; i < n; ++i) {
            const float f = (float)value(i);
            if (t == DGS_F32) ((float *)store.get())[i] = f;
            else if (t == DGS_BF16) ((uint16_t *)store.get())[i] = (uint16_t)(__float_as_uint(f) >> 16);
            else {
                const _Float16 h = (_Float16)f;
                memcpy((uint16_t *)store.get() + i, &h, 2);
            }
            v[i] = read_as(t, store.get(), i);
        }
    }
    dgs_matrix view(uint64_t stride) { return dgs_matrix{store.get(), stride}; }
    const float *floats() const { return (const float *)store.get(); }
};

static int power_of(double v) { int e; frexp(v, &e); return e; }      // smallest e with |v| < 2^e

// Loss and gradients of x, W, bias and targets, against the definition.  Logits are off by what fp32's additions leave of `cols` products and, of
// fp32 operands, by 2^-22 of each value and 2^-50 of its row's largest (2^-42 where the rows of W lie within 2^8 of one another); lse is off by their softmax mean (a tenth more for what is not linear) and 2^-22 of its
// terms' exponents, a value of dz, relatively, by what its logit and lse are and 2^-20 for the exponential.  dz is held in 22 bits, with steps of 2^-50 (half of it here) of its row's power of two.  x and W in the
// gradients' products: 2^-22 and 2^-50 of the largest for fp32, nothing and 2^-40 for half and bfloat16; dx of bfloat16 takes 11 bits of dz.
static void head(const char *what, int type, uint32_t rows, uint32_t cols, uint32_t vocab, const Mat &x, const Mat &w, const Mat *bias)
{
    name = std::string(what) + " " + std::to_string(type) + " " + std::to_string(rows) + "x" + std::to_string(cols) + "x" + std::to_string(vocab);
    Mat dloss(DGS_F32, rows, [](uint64_t) { return normal(); }), dlse(DGS_F32, rows, [](uint64_t) { return 0.1 * normal(); });
    auto none = [](uint64_t) { return NAN; };
    Mat loss(DGS_F32, rows, none), lse(DGS_F32, rows, none), dx(type, rows * cols, none), dw(DGS_F32, vocab * cols, none), db(DGS_F32, vocab, none);
    std::vector<int32_t> targets(rows);
    for (uint32_t t = 0; t < rows; ++t) targets[t] = t % 5 == 3 ? -100 : (int32_t)(2 * (gen() % ((vocab + 1) / 2)));
    dgs_head_args a = {};
    a.rows = rows; a.cols = cols; a.vocab = vocab;
    a.type = type; a.target_bytes = 4;
    a.x = dgs_matrix{x.store.get(), cols}; a.weight = dgs_matrix{w.store.get(), cols};
    a.bias = bias ? bias->floats() : nullptr;
    a.targets = targets.data();
    a.loss = (float *)loss.store.get(); a.lse = (float *)lse.store.get();
    auto call = [&](int back) {
        with_workspace(dgs_head_workspace(&a, back), [&](void *ws, uint64_t n) {
            a.workspace = ws;
            a.workspace_bytes = n;
            return back ? dgs_head_backward(&a, nullptr) : dgs_head_forward(&a, nullptr);
        }, back ? "backward" : "forward");
    };
    call(0);
    std::vector<double> z(rows * vocab), dz(rows * vocab), terms(rows * vocab), far(vocab);
    double w_most = 0.0, x_most = 0.0;
    std::vector<double> w_row(vocab), x_row(rows), up(rows), power(rows);
    for (uint32_t v = 0; v < vocab; ++v)
        for (uint32_t c = 0; c < cols; ++c) w_row[v] = std::max(w_row[v], std::fabs(w.v[v * cols + c]));
    double w_least = INFINITY;
    for (double v : w_row) w_most = std::max(w_most, v), w_least = v > 0.0 ? std::min(w_least, v) : w_least;
    const int row_step = w_most > 0.0 && power_of(w_most) - power_of(w_least) <= 8 ? -42 : -50;
    for (uint32_t t = 0; t < rows; ++t) {
        double top = -INFINITY, sum = 0.0, off = 0.0;
        for (uint32_t c = 0; c < cols; ++c) x_row[t] = std::max(x_row[t], std::fabs(x.v[t * cols + c]));
        for (uint32_t v = 0; v < vocab; ++v) {
            double s = bias ? bias->v[v] : 0.0, m = std::fabs(s), least = 0.0;
            for (uint32_t c = 0; c < cols; ++c) {
                const double p = x.v[t * cols + c], q = w.v[v * cols + c];
                s += p * q;
                m += std::fabs(p * q);
                least += std::fabs(p) * w_row[v] + std::fabs(q) * x_row[t];
            }
            z[t * vocab + v] = s;
            top = std::max(top, s);
            far[v] = std::isinf(s) ? 0.0 : ldexp(m * (cols + 8), -24) + (type == DGS_F32 ? ldexp(m, -21) + ldexp(least, row_step) : 0.0);
        }
        for (uint32_t v = 0; v < vocab; ++v) sum += exp(z[t * vocab + v] - top);
        const double l = top + log(sum);
        for (uint32_t v = 0; v < vocab; ++v) off += 1.1 * exp(z[t * vocab + v] - l) * far[v];
        const bool counts = targets[t] >= 0;
        off += ldexp(std::fabs(l) + 40.0, -22);
        near(read_as(DGS_F32, lse.store.get(), t), l, off, "lse", t);
        near(read_as(DGS_F32, loss.store.get(), t), counts ? l - z[t * vocab + targets[t]] : 0.0, counts ? off + far[targets[t]] : 0.0, "loss", t);
        up[t] = counts ? dloss.v[t] : 0.0;
        power[t] = power_of(std::max(std::fabs(up[t]), std::fabs(up[t] + dlse.v[t])));
        for (uint32_t v = 0; v < vocab; ++v) {
            const double p = (up[t] + dlse.v[t]) * exp(z[t * vocab + v] - l), one = (long)v == targets[t] ? up[t] : 0.0;
            dz[t * vocab + v] = p - one;
            terms[t * vocab + v] = std::fabs(p) * (off + far[v] + ldexp(1.0, -20)) + (std::fabs(p) + std::fabs(one)) * ldexp(1.0, -22) + ldexp(1.0, (int)power[t] - 50);
        }
        x_most = std::max(x_most, x_row[t] * ldexp(1.0, (int)power[t]));
    }
    a.dloss = dloss.floats();
    a.dlse = dlse.floats();
    a.dx = dx.view(cols);
    a.dweight = (float *)dw.store.get();
    a.dweight_stride = cols;
    a.dbias = (float *)db.store.get();
    call(1);
    const double held = type == DGS_F32 ? ldexp(1.0, -22) : 0.0;
    const int lost = type == DGS_F32 ? -50 : -40;
    for (uint32_t t = 0; t < rows; ++t)
        for (uint32_t c = 0; c < cols; ++c) {
            double s = 0.0, off = 0.0;
            for (uint32_t v = 0; v < vocab; ++v) {
                const double d = std::fabs(dz[t * vocab + v]), q = std::fabs(w.v[v * cols + c]);
                s += dz[t * vocab + v] * w.v[v * cols + c];
                off += terms[t * vocab + v] * q + d * (q * (held + ldexp((double)vocab, -24)) + ldexp(w_most, lost));
                if (type != DGS_F32) off += ldexp(d * q, -11) + ldexp(q, (int)power[t] - 39);
            }
            near(read_as(type, dx.store.get(), t * cols + c), s, off + std::fabs(s) * half_step(type) + (type == DGS_F16 ? ldexp(1.0, -25) : 0.0), "dx", t, c);
        }
    for (uint32_t v = 0; v < vocab; ++v) {
        double s = 0.0, off = 0.0;
        for (uint32_t t = 0; t < rows; ++t) s += dz[t * vocab + v], off += terms[t * vocab + v] + ldexp(std::fabs(dz[t * vocab + v]) * rows, -24);
        near(read_as(DGS_F32, db.store.get(), v), s, off, "dbias", v);
        for (uint32_t c = 0; c < cols; ++c) {
            s = off = 0.0;
            for (uint32_t t = 0; t < rows; ++t) {
                const double d = std::fabs(dz[t * vocab + v]), p = std::fabs(x.v[t * cols + c]);
                s += dz[t * vocab + v] * x.v[t * cols + c];
                off += terms[t * vocab + v] * p + d * (p * (held + ldexp((double)rows, -24)) + ldexp(x_most, lost - (int)power[t]));
            }
            near(read_as(DGS_F32, dw.store.get(), v * cols + c), s, off, "dweight", v, c);
        }
    }
}

// Half of the entries (no targets) lowered by their bias, to softmax of 2^-20 down to 2^-44: their weights' gradients keep their bits.
static void improbable()
{
    for (int type = 0; type < 3; ++type)
        for (double by : {10.0, 15.0, 20.0, 25.0}) {
            const uint32_t rows = by == 15.0 ? 20 : 40, cols = 64, vocab = 200;
            Mat x(type, rows * cols, [](uint64_t) { return normal(); }), w(type, vocab * cols, [](uint64_t) { return normal() / 8; });
            Mat bias(DGS_F32, vocab, [&](uint64_t v) { return v & 1 ? -by : 0.0; });
            head("improbable", type, rows, cols, vocab, x, w, &bias);
        }
}

// fp32: one entry of W far above the others, in a column where x is 0: what is small beside it decides about all
// logits but its own, which a bias takes out.  (From 33 rows on
// operands are held in halves; up to 32 they are read as they are.)
static void unlike()
{
    for (uint32_t rows : {32u, 33u, 70u})
        for (double far : {1e9, 1e12, 1e25}) {
            const uint32_t cols = 16, vocab = 64;
            Mat x(DGS_F32, rows * cols, [&](uint64_t i) { return i % cols == 5 ? 0.0 : normal(); });
            Mat w(DGS_F32, vocab * cols, [&](uint64_t i) { return i == 7 * cols + 5 ? far : normal(); });
            Mat bias(DGS_F32, vocab, [](uint64_t v) { return v == 7 ? -INFINITY : 0.0; });
            head("outlier", DGS_F32, rows, cols, vocab, x, w, &bias);
            if (far > 1e9) continue;
            // (x's columns 8 to 15 are 0 but in the odd rows, W's are large; entries take their logits from small numbers or large ones)
            Mat y(DGS_F32, rows * cols, [&](uint64_t i) { return i % cols < 8 ? normal() : i / cols % 2 ? normal() / far : 0.0; });
            Mat u(DGS_F32, vocab * cols, [&](uint64_t i) { return i % cols < 8 ? normal() : i / cols % 3 == 0 ? normal() * far : 0.0; });
            head("unlike columns", DGS_F32, rows, cols, vocab, y, u, nullptr);
        }
    // rows of W up to 2^8 and 2^9 apart, some of them zeros: dx and logits from one copy, and from one each
    for (int apart : {0, 8, 9, 60}) {
        const uint32_t rows = 40, cols = 24, vocab = 70;
        Mat x(DGS_F32, rows * cols, [&](uint64_t) { return normal(); });
        Mat w(DGS_F32, vocab * cols, [&](uint64_t i) { return i / cols % 5 == 2 ? 0.0 : ldexp(1.0 + (double)gen() / 4294967296.0, i / cols % 2 ? -apart : 0) * (i % 3 ? 0.3 : -0.3); });
        head(("apart by 2^" + std::to_string(apart)).c_str(), DGS_F32, rows, cols, vocab, x, w, nullptr);
    }
    Mat x(DGS_F32, 40 * 8, [&](uint64_t) { return normal(); }), zeros(DGS_F32, 50 * 8, [](uint64_t) { return 0.0; });
    head("zeros", DGS_F32, 40, 8, 50, x, zeros, nullptr);
}

int main(int, char **argv)
{
    const std::string what = argv[1];
    if (what == "coefficients") coefficients();
    if (what == "improbable") improbable();
    if (what == "unlike") unlike();
    printf("%llu values as expected\n", (unsigned long long)checks);
    return 0;
}
