"""The training blocks (paper_1910_10929_amd.blocks) against plain computations in 64 bits.

Tolerances.  A value that a kernel computes in fp32 and rounds once to its type differs from the exact one by at most half a
unit of the type, HALF[type] times its size, plus what fp32 leaves on the way: every intermediate is off by at most EPS = 2^-24 of
the largest number that went into it, some forty times over (a lane adds eight values, six joins make a wavefront, sixteen a
team, and the arithmetic around it), so 64 EPS of that size is allowed.  Column sums of n rows add a rounding a row, which
partial sums in a random order let grow with the root of n: 8 sqrt(n) EPS of the terms' 2-norm, and 64 EPS of the largest.
Whole numbers have no tolerance."""
import numpy as np
import pytest

from paper_1910_10929_amd import blocks, dgs

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"
EPS = 2.0 ** -24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
D = torch.float64


@pytest.fixture(scope="module", autouse=True)
def built():
    assert torch.cuda.is_available()
    dgs.lib()


class Make:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def __call__(self, rows, cols, dtype=F32, pad=0, scale=1.0, shift=0):
        """Normal values in the first columns of longer rows, `shift` elements into their buffer."""
        n = rows * (cols + pad) + shift
        t = torch.full((max(n, 1),), float("nan"), dtype=dtype, device=DEV)[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        t.copy_(torch.randn(rows, cols, device=DEV, generator=self.g) * scale)
        return t

    def vector(self, n, mean=1.0, dev=0.2, odd=1):
        t = torch.empty(n + odd, device=DEV)[odd:]
        t.copy_(mean + dev * torch.randn(n, device=DEV, generator=self.g))
        return t


def assert_near(got, want, size, what, dtype=None, extra=0.0):
    """|got - want| <= half a unit of the type + 64 EPS size + extra, everywhere."""
    dtype = dtype or got.dtype
    tol = HALF[dtype] * want.abs() + 64 * EPS * size + extra
    if dtype == F16:
        tol = tol + 2.0 ** -25      # (its smallest numbers have a fixed unit)
    bad = ~((got.to(D) - want).abs() <= tol)
    if bool(bad.any()):
        i = int(bad.reshape(-1).nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got.reshape(-1)[i].item()} != "
                             f"{want.reshape(-1)[i].item()} within {tol.expand_as(want).reshape(-1)[i].item()}")


def norm64(v, kind, eps):
    if kind is None:
        z = torch.zeros(v.shape[0], 1, dtype=D, device=DEV)
        return v, z, z
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros(v.shape[0], 1, dtype=D, device=DEV)
    rstd = 1.0 / ((v - mean).square().mean(1, keepdim=True) + eps).sqrt()
    return (v - mean) * rstd, mean, rstd


def values64(c):
    byte = c.exps.to(D).repeat_interleave(32, 1)[:, :c.cols]
    return torch.where(byte == 255, float("nan"), torch.exp2(byte - 127)) * c.codes.to(D)


def gates64(gate, per, rows):
    return 1.0 if gate is None else gate.to(D).repeat_interleave(per, 0)[:rows]


# rows, cols, stream, type, post, pre, biases, rows for each gate row, gate type, padding
EDGES = [
    (1, 1, F32, F32, "rms", "layer", True, 0, F32, 0),
    (3, 5, BF16, BF16, "layer", "rms", False, 2, BF16, 1),
    (70, 7, F32, F16, "layer", "layer", True, 1, F16, 0),
    (33, 8, F16, F16, "rms", "rms", True, 33, F32, 3),
    (1000, 31, F32, BF16, "layer", "layer", True, 7, BF16, 0),
    (1, 768, BF16, BF16, "layer", "layer", True, 0, F32, 0),
    (300, 768, F32, BF16, "layer", "layer", True, 64, BF16, 0),
    (517, 512, BF16, BF16, "rms", "rms", False, 1, BF16, 8),
    (130, 513, F16, F16, "layer", "rms", True, 130, F32, 3),
    (40, 1001, F32, F32, "layer", "rms", True, 37, F32, 5),
    (9000, 64, F32, F32, "rms", "layer", True, 32, F32, 0),
    (5000, 96, BF16, BF16, "rms", "rms", True, 2, BF16, 0),
    (64, 1536, BF16, BF16, None, "rms", False, 16, BF16, 0),
    (29, 2056, F32, F16, "rms", None, True, 0, F32, 1),
    (600, 4096, BF16, BF16, "rms", "rms", False, 600, F32, 0),
    (17, 4420, F16, F16, "layer", "layer", True, 1, F16, 0),
    (12, 8192, F32, BF16, "layer", "rms", True, 5, BF16, 0),
    (7, 10001, BF16, BF16, "layer", "layer", True, 3, BF16, 1),
    (3, 16384, F32, F32, "rms", "layer", True, 2, F32, 0),
]


class Case:
    """An edge, its inputs, and the forward pass in 64 bits."""

    def __init__(self, case, seed=0, branch=True):
        (self.rows, self.cols, self.stream, self.type, self.post, self.pre, bias, self.per, gate_type, self.pad) = case
        m = self.make = Make(seed + 13 * self.rows + self.cols)
        rows, cols, pad = self.rows, self.cols, self.pad
        if not branch:
            self.post, self.per = None, 0
        self.skip, self.branch = 1.25, 0.75
        self.x = m(rows, cols, self.stream, pad, 2.0, shift=1)
        self.f = m(rows, cols, self.type, pad) if branch else None
        self.gate = m((rows + self.per - 1) // self.per, cols, gate_type, pad) if self.per else None
        v = {}
        for name in ("post", "pre"):
            if getattr(self, name):
                v[name + "_weight"] = m.vector(cols)
                if bias:
                    v[name + "_bias"] = m.vector(cols, 0.0, 0.5)
        self.vectors = v
        self.edge = blocks.Edge(cols, post=self.post, pre=self.pre, skip_scale=self.skip, branch_scale=self.branch, eps=1e-4, **v)
        self.d = {k: t.to(D) for k, t in v.items()}

    def w(self, name, default):
        return self.d.get(name, torch.full((self.cols,), default, dtype=D, device=DEV))

    def forward64(self, x=None, f=None, gate=None, d=None):
        x = self.x.to(D) if x is None else x
        if self.f is None:
            xo, fh, fm, fr = x, None, torch.zeros(self.rows, 1, dtype=D, device=DEV), torch.zeros(self.rows, 1, dtype=D, device=DEV)
        else:
            fh, fm, fr = norm64(self.f.to(D) if f is None else f, self.post, 1e-4)
            g = gates64(self.gate, self.per, self.rows) if gate is None else gate.repeat_interleave(self.per, 0)[:self.rows]
            w = lambda n, v: (d or self.d).get(n, self.w(n, v))  # noqa: E731
            xo = self.skip * x + self.branch * g * (fh * w("post_weight", 1.0) + w("post_bias", 0.0))
        xh, xm, xr = norm64(xo, self.pre, 1e-4)
        w = lambda n, v: (d or self.d).get(n, self.w(n, v))  # noqa: E731
        u = xh * w("pre_weight", 1.0) + w("pre_bias", 0.0) if self.pre else None
        return xo, u, fh, xh, torch.cat([fm, fr, xm, xr], 1)


def check_codes(c, want, size, what):
    """Codes of computed values: nearest to them but for what fp32 leaves, in the run's own step."""
    step = torch.exp2(c.exps.to(D) - 127).repeat_interleave(32, 1)[:, :c.cols]
    assert bool(((values64(c) - want).abs() <= 0.5 * step + 64 * EPS * size).all()), what
    top = torch.nn.functional.pad(want.abs(), (0, c.exps.shape[1] * 32 - c.cols)).view(want.shape[0], -1, 32).amax(2)
    each = torch.exp2(c.exps.to(D) - 127)
    slack = 64 * EPS * size.max() if isinstance(size, torch.Tensor) else 64 * EPS * size
    assert bool((top < 127.5 * each + slack).all()) and bool(((top >= 63.75 * each - slack) | (c.exps == 1)).all()), what


@pytest.mark.parametrize("branch", [True, False])
@pytest.mark.parametrize("case", EDGES, ids=lambda c: f"{c[0]}x{c[1]}")
def test_edge_forward(case, branch):
    c = Case(case, branch=branch)
    if not branch and c.pre is None:
        pytest.skip("nothing to compute")
    xo, u, fh, xh, stats = c.forward64()
    saved = blocks.Saved(c.rows, c.cols, device=DEV)
    got_x, got_u = c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=c.per or None, save=saved)
    # without saving, and into rows of longer ones: the same bits
    again_x, again_u = c.make(c.rows, c.cols, c.stream, 5) if branch else None, c.make(c.rows, c.cols, c.type if branch else c.stream, 7)
    c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=c.per or None, x_out=again_x, u=again_u if c.pre else None)
    size_x = (c.skip * c.x.to(D)).abs() + (xo - c.skip * c.x.to(D)).abs() if branch else xo.abs()
    if branch:
        size_f = (fh * c.w("post_weight", 1.0)).abs() + c.w("post_bias", 0.0).abs()
        size_x = size_x + gates64(c.gate, c.per, c.rows) * size_f if c.gate is None else size_x + gates64(c.gate, c.per, c.rows).abs() * size_f
        assert_near(got_x, xo, size_x, "x_out")
        assert torch.equal(got_x, again_x)
        if c.post:
            top = fh.abs().amax(1, keepdim=True)
            check_codes(saved.post, fh, top + 1, "post codes")
        else:
            check_codes(saved.post, c.f.to(D), torch.zeros((), dtype=D, device=DEV), "post codes")
    else:
        assert got_x is c.x
    if c.pre:
        top = xh.abs().amax(1, keepdim=True) + stats[:, 3:4] * size_x.amax(1, keepdim=True)
        assert_near(got_u, u, top * c.w("pre_weight", 1.0).abs() + c.w("pre_bias", 0.0).abs(), "u")
        assert torch.equal(got_u, again_u)
        check_codes(saved.pre, xh, top, "pre codes")
    big = torch.cat([(c.f if branch else c.x).to(D).abs().amax(1, keepdim=True)] * 2 + [size_x.amax(1, keepdim=True)] * 2, 1)
    rel = torch.cat([stats[:, 0:1] * 0 + 1, stats[:, 1:2].square(), stats[:, 2:3] * 0 + 1, stats[:, 3:4].square()], 1)
    assert_near(saved.stats, stats, big * rel + stats.abs(), "stats")


def backward64(c, d_in, u_in, fh, xh, stats):
    rows = c.rows

    def through(g, h, rstd, kind):
        if kind is None:
            return g
        g = g - h * (g * h).mean(1, keepdim=True) - (g.mean(1, keepdim=True) if kind == "layer" else 0.0)
        return rstd * g
    d = d_in.to(D) if d_in is not None else torch.zeros(rows, c.cols, dtype=D, device=DEV)
    out = {}
    if u_in is not None:
        u = u_in.to(D)
        out["pre_weight"], out["pre_bias"] = (u * xh).sum(0), u.sum(0)
        out["size_pre_weight"], out["size_pre_bias"] = (u * xh), u
        d = d + through(u * c.w("pre_weight", 1.0), xh, stats[:, 3:4], c.pre)
    out["dx"] = c.skip * d
    if c.f is not None:
        n = fh * c.w("post_weight", 1.0) + c.w("post_bias", 0.0)
        out["n"] = n
        if c.gate is not None:
            each = c.branch * d * n
            gates = c.gate.shape[0]
            which = torch.arange(rows, device=DEV) // c.per
            out["dgate"] = torch.zeros(gates, c.cols, dtype=D, device=DEV).index_add_(0, which, each)
            out["size_dgate"] = torch.zeros(gates, c.cols, dtype=D, device=DEV).index_add_(0, which, each.square()).sqrt()
        m = c.branch * gates64(c.gate, c.per, rows) * d
        out["post_weight"], out["post_bias"] = (m * fh).sum(0), m.sum(0)
        out["size_post_weight"], out["size_post_bias"] = m * fh, m
        out["df"] = through(m * c.w("post_weight", 1.0), fh, stats[:, 1:2], c.post)
        out["m"] = m
    return out


def run_backward(c, saved, d_in, u_in, accumulate=False, start=0.0, **more):
    """The gradients a call gives, parameter gradients in vectors at odd places that held `start`."""
    grads = {}
    for name in ("post_weight", "post_bias", "pre_weight", "pre_bias"):
        if name.startswith("post") and c.f is None or name.startswith("pre") and u_in is None:
            continue
        t = torch.full((c.cols + 3,), start, device=DEV)
        grads[name] = t[3:]
    if c.gate is not None:
        grads["dgate"] = torch.full_like(c.gate, start)
    dx, df = c.edge.backward(saved, dx_out=d_in, du=u_in, gate=c.gate, rows_per_gate=c.per or None, dgate=grads.get("dgate"),
                             post_weight_grad=grads.get("post_weight"), post_bias_grad=grads.get("post_bias"),
                             pre_weight_grad=grads.get("pre_weight"), pre_bias_grad=grads.get("pre_bias"), accumulate=accumulate, **more)
    grads["dx"] = dx
    if df is not None:
        grads["df"] = df
    return grads


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("case", EDGES, ids=lambda c: f"{c[0]}x{c[1]}")
def test_edge_backward(case, coded):
    c = Case(case, seed=5)
    rows, cols = c.rows, c.cols
    saved = blocks.Saved(rows, cols, device=DEV, checkpoints=coded)
    xo, _ = c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=c.per or None, save=saved)
    d_in = c.make(rows, cols, c.stream, c.pad, shift=1)
    u_in = c.make(rows, cols, c.type, c.pad) if c.pre else None
    stats = saved.stats.to(D)
    if coded:
        fh, xh = values64(saved.post), values64(saved.pre) if c.pre else None
    else:
        fh = (c.f.to(D) - stats[:, 0:1]) * stats[:, 1:2] if c.post else c.f.to(D)
        xh = (xo.to(D) - stats[:, 2:3]) * stats[:, 3:4] if c.pre else None
    want = backward64(c, d_in, u_in, fh, xh, stats)
    accumulate = rows % 2 == 1
    got = run_backward(c, saved, d_in, u_in, accumulate=accumulate, start=0.5 if accumulate else float("nan"))
    # the largest number that goes into a row's gradients
    top = d_in.to(D).abs().amax(1, keepdim=True)
    if u_in is not None:
        top = top + (stats[:, 3:4] * (u_in.to(D) * c.w("pre_weight", 1.0)).abs().amax(1, keepdim=True)
                     * (1 + xh.abs().amax(1, keepdim=True).square() + stats[:, 3:4] * 0))
    assert_near(got["dx"], want["dx"], c.skip * top, "dx")
    top_m = top * c.branch * (gates64(c.gate, c.per, rows).abs().amax(1, keepdim=True) if c.gate is not None else 1.0)
    rstd = stats[:, 1:2] if c.post else 1.0
    assert_near(got["df"], want["df"], rstd * top_m * (c.w("post_weight", 1.0).abs().max()) * (1 + fh.abs().amax(1, keepdim=True).square()), "df")
    n_sqrt = 8 * rows ** 0.5
    for name, got_sum in got.items():
        if name in ("dx", "df", "dgate"):
            continue
        terms = want["size_" + name]
        size = terms.square().sum(0).sqrt()
        base = 0.5 if accumulate else 0.0
        err_in = (top_m if name.startswith("post") else top * 0).to(D) * (fh.abs() if name == "post_weight" else 1.0)
        assert_near(got_sum, want[name] + base, terms.abs().amax(0) + base, name, extra=n_sqrt * EPS * size + 64 * EPS * err_in.square().sum(0).sqrt())
    if c.gate is not None:
        adds = accumulate and c.gate.dtype == F32
        err_in = (c.branch * top * want["n"].abs())
        which = torch.arange(rows, device=DEV) // c.per
        err = torch.zeros_like(want["dgate"]).index_add_(0, which, err_in.square()).sqrt()
        assert_near(got["dgate"], want["dgate"] + (0.5 if adds else 0.0), want["dgate"].abs() + 1.0 * adds, "dgate",
                    extra=8 * min(rows, c.per) ** 0.5 * EPS * want["size_dgate"] + 64 * EPS * err)


@pytest.mark.parametrize("kinds", [("layer", "layer"), ("rms", "layer"), (None, "rms"), ("rms", None)])
def test_edge_gradient_against_differences(kinds):
    """<gradient, direction> against a central difference of the loss sum(x_out D) + sum(u U) in 64 bits, step 1e-5: it is off by
    some 1e-10 of the loss's third derivative; fp32 gradients of 24 x 40 values, at most 1e-4 of the sums that they go into."""
    rows, cols = 24, 40
    c = Case((rows, cols, F32, F32, kinds[0], kinds[1], True, 5, F32, 0), seed=9)
    saved = blocks.Saved(rows, cols, device=DEV, checkpoints=False)
    c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=c.per, save=saved)
    d_in, u_in = c.make(rows, cols), c.make(rows, cols) if c.pre else None
    got = run_backward(c, saved, d_in, u_in)
    inputs = {"dx": ("x", c.x), "df": ("f", c.f), "dgate": ("gate", c.gate)}
    inputs.update({name: (name, v) for name, v in c.vectors.items()})

    def loss(name, moved):
        args = {"x": c.x.to(D), "f": c.f.to(D), "gate": c.gate.to(D)}
        d = dict(c.d)
        (args if name in args else d)[name] = moved
        xo, u, *_ = c.forward64(**args, d=d)
        return float((xo * d_in.to(D)).sum() + ((u * u_in.to(D)).sum() if u is not None else 0.0))

    for key, (name, value) in inputs.items():
        for k in range(3):
            direction = torch.randn(value.shape, dtype=D, device=DEV, generator=c.make.g)
            h = 1e-5
            want = (loss(name, value.to(D) + h * direction) - loss(name, value.to(D) - h * direction)) / (2 * h)
            have = float((got[key].to(D) * direction).sum())
            size = float((got[key].to(D) * direction).square().sum().sqrt())
            assert abs(have - want) <= 1e-4 * (size + 1.0), (key, have, want)


def test_edge_without_arriving_gradients():
    """Either gradient may be absent: the same as zeros."""
    c = Case((50, 96, F32, BF16, "rms", "layer", True, 7, BF16, 0))
    saved = blocks.Saved(50, 96, device=DEV)
    c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=7, save=saved)
    d, u = c.make(50, 96, F32), c.make(50, 96, BF16)
    dx = torch.empty(50, 96, device=DEV)
    for have, zeros in ((dict(d_in=d, u_in=None), dict(d_in=d, u_in=torch.zeros_like(u))), (dict(d_in=None, u_in=u), dict(d_in=torch.zeros_like(d), u_in=u))):
        a, b = run_backward(c, saved, dx=dx, **have) if have["d_in"] is None else run_backward(c, saved, df=torch.empty_like(u), **have), run_backward(c, saved, **zeros)
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_edge_in_place_and_repeatable():
    for case in ((700, 768, BF16, BF16, "layer", "rms", True, 100, BF16, 3), (300, 1001, F16, F16, "rms", "layer", True, 1, F16, 0),
                 (64, 6000, F32, F32, "layer", "layer", True, 64, F32, 0)):
        c = Case(case)
        saved, saved2 = blocks.Saved(c.rows, c.cols, device=DEV), blocks.Saved(c.rows, c.cols, device=DEV)
        xo, u = c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=c.per, save=saved)
        x2, f2 = c.x.clone(), c.f.clone()
        xo2, u2 = c.edge.forward(x2, f2, gate=c.gate, rows_per_gate=c.per, x_out=x2, u=f2, save=saved2)
        assert xo2 is x2 and u2 is f2 and torch.equal(xo, x2) and torch.equal(u, f2)
        for a, b in ((saved.post, saved2.post), (saved.pre, saved2.pre)):
            assert torch.equal(a.codes, b.codes) and torch.equal(a.exps, b.exps)
        d, du = c.make(c.rows, c.cols, c.stream), c.make(c.rows, c.cols, c.type)
        one = run_backward(c, saved, d, du)
        two = run_backward(c, saved, d, du)
        d2, du2 = d.clone(), du.clone()
        three = run_backward(c, saved, d2, du2, dx=d2, df=du2)
        for k in one:
            assert torch.equal(one[k], two[k]) and torch.equal(one[k], three[k]), k


def test_edge_rows_do_not_meet():
    """Rows of infinities, NaN, zeros and large values leave the others as they are; a row of zeros is finite."""
    rows, cols = 40, 100
    c = Case((rows, cols, F32, F32, "layer", "rms", True, 0, F32, 0))
    plain = c.edge.forward(c.x, c.f)
    x, f = c.x.clone(), c.f.clone()
    f[3, 50] = float("nan")
    f[7, 99] = float("inf")
    x[11] = -float("inf")
    f[12], x[12] = 0.0, 0.0
    x[13] *= 1e15
    saved = blocks.Saved(rows, cols, device=DEV)
    xo, u = c.edge.forward(x, f, save=saved)
    same = [r for r in range(rows) if r not in (3, 7, 11, 12, 13)]
    assert torch.equal(xo[same], plain[0][same]) and torch.equal(u[same], plain[1][same])
    assert bool(torch.isnan(u[3]).all()) and bool(torch.isnan(xo[7, 99]))
    assert bool(torch.isfinite(xo[12:14]).all()) and bool(torch.isfinite(u[12:14]).all())
    assert bool((saved.post.exps[3] == 255).all()) and bool((saved.post.codes[3] == 0).all())
    assert bool((saved.pre.exps[same] != 255).all())


def test_no_rows():
    e = blocks.Edge(64, post="rms", pre="layer")
    x = torch.empty(0, 64, device=DEV)
    saved = blocks.Saved(0, 64, device=DEV)
    xo, u = e.forward(x, x.clone(), save=saved)
    assert xo.shape == u.shape == (0, 64)
    g = [torch.full((64,), 3.0, device=DEV) for _ in range(2)]
    e.backward(saved, dx_out=x, du=x, post_weight_grad=g[0], pre_weight_grad=g[1], accumulate=True)
    assert all(bool((t == 3.0).all()) for t in g)
    e.backward(saved, dx_out=x, du=x, post_weight_grad=g[0], pre_weight_grad=g[1])
    assert all(bool((t == 0.0).all()) for t in g)
    c = blocks.Checkpoint(0, 64, device=DEV).encode(x)
    assert c.decode().shape == (0, 64)
    dw = torch.full((5, 64), 3.0, device=DEV)
    db = torch.full((5,), 3.0, device=DEV)
    blocks.weight_grad(torch.empty(0, 5, device=DEV), c, dw, db, accumulate=True)
    assert bool((dw == 3.0).all()) and bool((db == 3.0).all())
    blocks.weight_grad(torch.empty(0, 5, device=DEV), c, dw, db, shift=torch.ones(64, device=DEV))
    assert bool((dw == 0.0).all()) and bool((db == 0.0).all())


# ----------------------------------------------------------------------------
# checkpoints
# ----------------------------------------------------------------------------

def codes_of(x):
    """The definition, on the host in 64 bits: codes and bytes of a float64 array."""
    rows, cols = x.shape
    runs = (cols + 31) // 32
    p = np.zeros((rows, runs * 32))
    p[:, :cols] = x
    p = p.reshape(rows, runs, 32)
    q, byte = np.zeros(p.shape), np.zeros((rows, runs))
    for r in range(rows):
        for k in range(runs):
            v = p[r, k]
            if not np.isfinite(v).all():
                byte[r, k] = 255
                continue
            e = -126
            while e < 121 and np.abs(v).max() >= np.ldexp(127.5, e):
                e += 1
            byte[r, k] = e + 127
            q[r, k] = np.clip(np.rint(np.ldexp(v, -e)), -127, 127)      # (rint: halfway cases to even)
    return q.reshape(rows, -1)[:, :cols], byte


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows, cols, pad", [(1, 1, 0), (2, 7, 1), (3, 33, 0), (5, 64, 3), (4, 100, 8), (3, 1000, 0)])
def test_checkpoint_is_the_definition(rows, cols, pad, dtype):
    m = Make(rows * 1000 + cols)
    x = m(rows, cols, dtype, pad, 1.0, shift=1)
    x *= torch.exp2(torch.randint(-8, 9, (rows, 1), device=DEV, generator=m.g).to(dtype))
    if cols > 2:
        x[0, 0], x[0, 1] = 127.5, -0.5      # a power more is needed; halfway between codes
    c = blocks.Checkpoint(rows, cols, DEV).encode(x)
    q, byte = codes_of(x.to(D).cpu().numpy())
    np.testing.assert_array_equal(c.codes.cpu().numpy(), q)
    np.testing.assert_array_equal(c.exps.cpu().numpy(), byte)
    assert torch.equal(c.decode(dtype=F32).to(D), values64(c)) and torch.equal(c.decode(dtype=BF16).to(D), values64(c))
    scale, shift = m.vector(cols), m.vector(cols, 0.0)
    for out in (F32, F16, BF16):
        want = values64(c) * scale.to(D) + shift.to(D)
        assert_near(c.decode(m(rows, cols, out, 3), scale=scale, shift=shift), want, values64(c).abs() * scale.abs() + shift.abs(), "decode")
        want = values64(c) * scale.to(D)
        assert_near(c.decode(dtype=out, scale=scale), want, want.abs(), "decode")


def test_checkpoint_of_extremes():
    big = torch.finfo(F32).max
    inf, nan = float("inf"), float("nan")
    x = torch.zeros(12, 64, device=DEV)
    x[0, 3], x[1, 40], x[2, 5] = nan, inf, -inf
    x[3] = -0.0
    x[4, :4] = torch.tensor([big, -big, 1.0, 2.0 ** 121])
    x[5, :3] = torch.tensor([2.0 ** -149, -2.0 ** -140, 2.0 ** -126])
    x[6, :3] = torch.tensor([2.0 ** -126 * 127, 2.0 ** -126 * 0.5, 2.0 ** -127])
    x[7, :4] = torch.tensor([127.5, 126.5, 0.5, 1.5])
    x[8, :4] = torch.tensor([127.49999, 126.5, 0.5, -2.5])
    x[9, :2] = torch.tensor([1.5 * 2.0 ** 127, 2.0 ** 120])
    x[10, 0] = 65504.0
    x[11, 32] = 2.0 ** 121 * 127.5
    c = blocks.Checkpoint(12, 64, DEV).encode(x)
    q, byte = codes_of(x.to(D).cpu().numpy())
    np.testing.assert_array_equal(c.codes.cpu().numpy(), q)
    np.testing.assert_array_equal(c.exps.cpu().numpy(), byte)
    v = c.decode()
    assert bool(torch.isnan(v[0, :32]).all()) and bool((v[0, 32:] == 0).all()) and bool(torch.isfinite(v[3:]).all())
    # what comes near the largest half stays finite
    h = torch.full((2, 32), 65504.0, dtype=F16, device=DEV)
    h[1] = -65504.0
    got = blocks.Checkpoint(2, 32, DEV).encode(h).decode(dtype=F16)
    assert torch.equal(got, h)


# ----------------------------------------------------------------------------
# the weight gradient
# ----------------------------------------------------------------------------

# rows, outs, cols: one row; few of everything; each kind of tile, whole and cut; several splits of the rows, uneven
GRADS = [(1, 1, 1), (1, 300, 200), (5, 8, 8), (20, 130, 70), (31, 64, 513), (32, 8, 8), (33, 9, 15), (64, 128, 128), (100, 7, 300), (257, 200, 6),
         (256, 256, 256), (300, 257, 300), (1000, 129, 65), (2049, 384, 128), (4100, 768, 768), (5000, 520, 264), (9000, 64, 96), (700, 2304, 768),
         (513, 4096, 2048)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows, outs, cols", GRADS)
def test_weight_grad_of_whole_numbers(rows, outs, cols, dtype):
    """Small whole numbers times small powers of two: every product and every sum is exact in fp32, so the result is, whatever
    the order; each run of columns has powers of its own from row to row."""
    m = Make(rows + 3 * outs + 7 * cols)
    pad = cols % 3
    dy = m(rows, outs, dtype, pad, shift=1)
    dy.copy_(torch.randint(-3, 4, (rows, outs), device=DEV, generator=m.g))
    q = torch.randint(-15, 16, (rows, cols + pad), device=DEV, generator=m.g, dtype=torch.int32).to(torch.int8)[:, :cols]
    e = torch.randint(126, 129, (rows, (cols + 31) // 32 + pad), device=DEV, generator=m.g).to(torch.uint8)[:, :(cols + 31) // 32]
    c = blocks.Checkpoint.of(q, e)
    x = values64(c)
    want, want_db = dy.to(D).t() @ x, dy.to(D).sum(0)
    dw, db = torch.full((outs, cols + 5), float("nan"), device=DEV)[:, :cols], torch.full((outs,), float("nan"), device=DEV)
    blocks.weight_grad(dy, c, dw, db)
    assert torch.equal(dw.to(D), want) and torch.equal(db.to(D), want_db)
    # added to what is there, with a scale that is a power of two and a whole shift
    scale, shift = torch.exp2(torch.randint(0, 2, (cols,), device=DEV, generator=m.g).float()), torch.randint(-2, 3, (cols,), device=DEV, generator=m.g).float()
    blocks.weight_grad(dy, c, dw, db, scale=scale, shift=shift, accumulate=True)
    assert torch.equal(dw.to(D), want + want * scale.to(D) + want_db[:, None] * shift.to(D)) and torch.equal(db.to(D), 2 * want_db)
    blocks.weight_grad(dy, c, dw, scale=scale)
    assert torch.equal(dw.to(D), want * scale.to(D))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows, outs, cols", [(3, 40, 50), (100, 128, 130), (1024, 300, 256), (6000, 256, 512), (8192, 1024, 768),
                                              (600, 4096, 4096), (1100, 2300, 4001)])
def test_weight_grad(rows, outs, cols, dtype):
    """Against 64 bits.  Every product is exact; a sum of n of them is rounded n times, its partial sums in random signs are of
    the size of the terms' 2-norm."""
    m = Make(rows + outs)
    dy = m(rows, outs, dtype, 1, 0.01)
    c = blocks.Checkpoint(rows, cols, DEV).encode(m(rows, cols, F32, 0, 3.0))
    scale, shift = m.vector(cols), m.vector(cols, 0.0, 0.5)
    x, d = values64(c), dy.to(D)
    dw, db = torch.empty(outs, cols, device=DEV), torch.empty(outs, device=DEV)
    blocks.weight_grad(dy, c, dw, db, scale=scale, shift=shift)
    want_db = d.sum(0)
    want = (d.t() @ x) * scale.to(D) + want_db[:, None] * shift.to(D)
    size_db = d.square().sum(0).sqrt()
    size = (d.square().t() @ x.square()).sqrt() * scale.abs() + size_db[:, None] * shift.abs()
    n = 8 * rows ** 0.5 + 64
    assert bool(((dw.to(D) - want).abs() <= n * EPS * size).all())
    assert bool(((db.to(D) - want_db).abs() <= n * EPS * size_db).all())
    again = torch.empty_like(dw)
    blocks.weight_grad(dy, c, again, scale=scale, shift=shift)
    assert torch.equal(dw, again)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows", [20, 600])
def test_weight_grad_of_what_is_not_finite(rows, dtype):
    """An infinite or undefined gradient reaches its output's row alone, a run that reads as NaN its columns."""
    m = Make(1)
    dy = m(rows, 100, dtype)
    c = blocks.Checkpoint(rows, 160, DEV).encode(m(rows, 160).abs() + 0.5)
    base = torch.empty(100, 160, device=DEV)
    blocks.weight_grad(dy, c, base)
    dy[3, 7], dy[rows - 1, 64] = float("inf"), float("nan")
    got = torch.empty(100, 160, device=DEV)
    blocks.weight_grad(dy, c, got)
    others = [o for o in range(100) if o not in (7, 64)]
    assert torch.equal(got[others], base[others])
    assert bool(torch.isinf(got[7]).all()) and bool(torch.isnan(got[64]).all())
    dy[3, 7], dy[rows - 1, 64] = 1.0, 1.0
    blocks.weight_grad(dy, c, base)
    c.exps[5, 1] = 255
    blocks.weight_grad(dy, c, got)
    assert bool(torch.isnan(got[:, 32:64]).all()) and torch.equal(got[:, :32], base[:, :32]) and torch.equal(got[:, 64:], base[:, 64:])


# ----------------------------------------------------------------------------
# places beyond 32 bits, streams, graphs, the binding's checks
# ----------------------------------------------------------------------------

def test_rows_beyond_32_bits():
    """Matrices whose last rows begin more than 2^32 elements behind their first."""
    rows, cols, apart = 70_001, 40, 65_600
    room = torch.empty(rows * apart, dtype=torch.int8, device=DEV)
    half = torch.empty(rows * apart, dtype=BF16, device=DEV).view(rows, apart)[:, :cols]
    m = Make(3)
    small = m(rows, cols, BF16)
    half.copy_(small)
    codes = room.view(rows, apart)[:, :cols]
    c, s = blocks.Checkpoint(rows, cols, codes=codes, exps=torch.empty(rows, 2, dtype=torch.uint8, device=DEV)).encode(half), blocks.Checkpoint(rows, cols, DEV).encode(small)
    assert torch.equal(c.codes, s.codes) and torch.equal(c.exps, s.exps) and torch.equal(c.decode(dtype=BF16), s.decode(dtype=BF16))
    e = blocks.Edge(cols, post="rms", pre="layer")
    f = m(rows, cols, BF16)
    xo, u = e.forward(small, f)
    xo2, u2 = e.forward(half, f, x_out=half)
    assert torch.equal(xo, xo2) and torch.equal(u, u2)
    half.copy_(small)
    a, b = torch.empty(cols, cols, device=DEV), torch.empty(cols, cols, device=DEV)
    blocks.weight_grad(small, s, a)
    blocks.weight_grad(half, c, b)
    assert torch.equal(a, b)
    saved = blocks.Saved(rows, cols, device=DEV)
    e.forward(small, f, save=saved)
    far = blocks.Saved(rows, cols, stats=saved.stats, post=saved.post, pre=c)
    c.codes.copy_(saved.pre.codes)
    c.exps.copy_(saved.pre.exps)
    one, two = e.backward(saved, dx_out=small, du=f), e.backward(far, dx_out=half, du=f)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


def _step(c, dy, dw, db, grads, out):
    saved, x, f, gate = out["saved"], out["x"], out["f"], out["gate"]
    c.edge.forward(x, f, gate=gate, rows_per_gate=c.per, x_out=out["xo"], u=out["u"], save=saved)
    blocks.weight_grad(dy, saved.pre, dw, db, scale=c.edge.pre_weight, shift=c.edge.pre_bias, accumulate=True, workspace=out["ws"])
    c.edge.backward(saved, dx_out=out["xo"], du=out["u"], gate=gate, rows_per_gate=c.per, dx=out["dx"], df=out["df"], dgate=out["dg"],
                    post_weight_grad=grads[0], post_bias_grad=grads[1], pre_weight_grad=grads[2], pre_bias_grad=grads[3], accumulate=True,
                    workspace=out["ws"])


def _outs(c):
    out = {"saved": blocks.Saved(c.rows, c.cols, device=DEV), "x": c.x, "f": c.f, "gate": c.gate, "xo": torch.empty(c.rows, c.cols, dtype=c.stream, device=DEV),
           "u": torch.empty(c.rows, c.cols, dtype=c.type, device=DEV), "dx": torch.empty(c.rows, c.cols, dtype=c.stream, device=DEV),
           "df": torch.empty(c.rows, c.cols, dtype=c.type, device=DEV), "dg": torch.empty_like(c.gate),
           "ws": torch.empty(64 << 20, dtype=torch.uint8, device=DEV)}
    return out


def test_another_stream_and_a_graph():
    """On a side stream and replayed from a graph: the same bits as eagerly on the default stream, with other work between."""
    c = Case((600, 768, F32, BF16, "layer", "layer", True, 100, BF16, 0))
    dy = c.make(600, 256, BF16)
    results = []

    def fresh():
        return torch.zeros(256, 768, device=DEV), torch.zeros(256, device=DEV), [torch.zeros(768, device=DEV) for _ in range(4)], _outs(c)

    dw, db, grads, out = fresh()
    _step(c, dy, dw, db, grads, out)
    results.append([dw, db, *grads, out["dx"], out["df"], out["dg"], out["xo"], out["u"]])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    dw, db, grads, out = fresh()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(c, dy, dw, db, grads, out)
    side.synchronize()
    results.append([dw, db, *grads, out["dx"], out["df"], out["dg"], out["xo"], out["u"]])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    dw, db, grads, out = fresh()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        _step(c, dy, dw, db, grads, out)
    for replay in range(4):
        for t in (dw, db, *grads):
            t.zero_()
        for t in (out["dx"], out["df"], out["dg"], out["xo"], out["u"]):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results[0], [dw, db, *grads, out["dx"], out["df"], out["dg"], out["xo"], out["u"]]):
            assert torch.equal(a, b), replay
        assert float(torch.randn(1000, device=DEV).sum()) != 0.0      # (other work in between)


def test_binding_refuses():
    x, f = torch.zeros(6, 32, device=DEV), torch.zeros(6, 32, device=DEV, dtype=BF16)
    w = torch.ones(32, device=DEV)
    e = blocks.Edge(32, post="rms", pre="layer", pre_weight=w)
    saved = blocks.Saved(6, 32, device=DEV)
    c = blocks.Checkpoint(6, 32, DEV).encode(x)
    dw = torch.zeros(4, 32, device=DEV)
    dy = torch.zeros(6, 4, device=DEV)
    bad = [
        lambda: blocks.Edge(32, pre="rms", pre_weight=w.half()), lambda: blocks.Edge(32, pre="rms", pre_weight=w[:31]),
        lambda: blocks.Edge(16, pre="rms", pre_weight=w[::2]), lambda: blocks.Edge(32, pre="rms", pre_weight=torch.ones(32)),
        lambda: e.forward(x[0], f), lambda: e.forward(x[:, :31], f), lambda: e.forward(x, f[:5]), lambda: e.forward(x.double(), f),
        lambda: e.forward(x, f.cpu()), lambda: e.forward(x.t().contiguous().t()[:, :32], f),
        lambda: e.forward(x, f, gate=f[:4]), lambda: e.forward(x, f, gate=f, rows_per_gate=2), lambda: e.forward(x, f, gate=f, rows_per_gate=0),
        lambda: e.forward(x, f, gate=f.half(), rows_per_gate=1), lambda: e.forward(x, f, x_out=f), lambda: e.forward(x, f, u=x),
        lambda: e.forward(x), lambda: e.forward(x, f, save=blocks.Saved(5, 32, device=DEV)), lambda: e.forward(x.expand(6, 32)[:1].expand(6, 32), f),
        lambda: blocks.Edge(32, post="rms").forward(x, f, u=f),
        lambda: e.backward(saved), lambda: e.backward(saved, dx_out=x[:5], du=f), lambda: e.backward(saved, dx_out=x, du=f, dx=f),
        lambda: e.backward(saved, dx_out=x, du=f, df=x), lambda: e.backward(saved, dx_out=x, du=f, dgate=f),
        lambda: e.backward(saved, dx_out=x, du=f, gate=f, dgate=x), lambda: e.backward(saved, dx_out=x, du=f, post_weight_grad=w.half()),
        lambda: e.backward(blocks.Saved(6, 32, stats=saved.stats, post=saved.post, x_out=x), dx_out=x, du=f),
        lambda: e.backward(saved, dx_out=x, du=f, workspace=torch.empty(16, dtype=torch.uint8, device=DEV)),
        lambda: blocks.Edge(32, post="rms").backward(saved, dx_out=x, du=f),
        lambda: blocks.Checkpoint.of(c.codes, c.exps[:, :0]), lambda: blocks.Checkpoint.of(c.exps, c.codes), lambda: c.encode(x[:5]),
        lambda: c.decode(out=x[:, :31]), lambda: c.decode(scale=w.half()), lambda: c.decode(shift=w[:5]), lambda: c.decode(dtype=torch.float64),
        lambda: blocks.weight_grad(dy[:5], c, dw), lambda: blocks.weight_grad(dy, c, dw.half()), lambda: blocks.weight_grad(dy, c, dw[:3]),
        lambda: blocks.weight_grad(dy, c, dw, db=w), lambda: blocks.weight_grad(dy, c, dw, scale=w[:5]), lambda: blocks.weight_grad(dy.long(), c, dw),
        lambda: blocks.weight_grad(dy, c, dw, workspace=torch.empty(16, dtype=torch.uint8, device=DEV)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(dgs.DgsError):
            call()
            raise AssertionError(f"call {i} was not refused")
    big = torch.zeros(2, 16385, device=DEV)
    with pytest.raises(dgs.DgsError) as err:
        blocks.Edge(16385, pre="rms").forward(big)
    assert err.value.code == dgs.DGS_ENOTSUP
    torch.cuda.synchronize()
