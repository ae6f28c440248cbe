"""Orthogonalised updates (blocks.orthogonalise) against the iteration in 64 bits.

Tolerances.  Small singular values grow by up to 3.4445 a step, and with them what rounding has put among them; how far a result may be
off so depends on the matrix.  `noisy` runs the iteration in 64 bits with a random error of the size that the kernels' formats allow
wherever they round: X by up to 2^-22 of a value (two halves), A and the polynomial without its diagonal by 2^-22 or, for bfloat16
results, 2^-11, of which products then take X too, and sums of n products by 2^-24 sqrt(n) of the terms' 2-norm (bounded by the
operands' norms).  A result may be three times as far off, in the 2-norm, as the worst of three such runs, plus half a step of its
type; single values six times as far, in units of the error's root mean square times the largest of 4.5 that a normal sample of this size
reaches."""
import pytest

from paper_1910_10929_amd import blocks, dgs

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"
F32, F16, BF16, D = torch.float32, torch.float16, torch.bfloat16, torch.float64
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module", autouse=True)
def built():
    assert torch.cuda.is_available()
    dgs.lib()


class Make:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, device=DEV, generator=self.g)

    def matrix(self, rows, cols, dtype=F32, kind="normal", pad=0, shift=0):
        if kind == "normal":
            m = self.normal(rows, cols)
        elif kind == "gradient":        # a sum over rows of a batch, channels of unlike scale
            m = (self.normal(rows, 2 * min(rows, cols)) * torch.exp(0.5 * self.normal(rows, 1))) @ (self.normal(2 * min(rows, cols), cols) * torch.exp(0.5 * self.normal(cols)))
        else:                           # a few directions far above the others
            m = self.normal(rows, 4) @ self.normal(4, cols) + 0.05 * self.normal(rows, cols)
        n = rows * (cols + pad) + shift
        t = torch.full((n,), float("nan"), dtype=dtype, device=DEV)[shift:].view(rows, cols + pad)[:, :cols]
        t.copy_(m * (0.01 if dtype != F16 else 0.1))
        return t


def exact(g, steps=5, eps=1e-7, coefficients=COEFFICIENTS):
    a, b, c = (torch.tensor(v, dtype=F32).to(D).item() for v in coefficients)
    x = g.to(D)
    x = x / (torch.linalg.vector_norm(x) + torch.tensor(eps, dtype=F32).to(D).item())
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for _ in range(steps):
        m = x @ x.t()
        x = a * x + (b * m + c * (m @ m)) @ x
    return x.t() if tall else x


def noisy(g, two, gen, steps=5):
    a, b, c = COEFFICIENTS
    short = 2.0 ** -22 if two else 2.0 ** -11

    def off(v, by):
        return v * (1.0 + by * (2.0 * torch.rand(v.shape, dtype=D, device=DEV, generator=gen) - 1.0))

    def product(p, q):
        terms = torch.sqrt((p * p) @ (q * q))
        return p @ q + 2.0 ** -24 * p.shape[1] ** 0.5 * terms * torch.randn(terms.shape, dtype=D, device=DEV, generator=gen)

    x = g.to(D)
    x = x / (torch.linalg.vector_norm(x) + 1e-7)
    x = x.t().contiguous() if x.shape[0] > x.shape[1] else x
    for _ in range(steps):
        x = off(x, 2.0 ** -22)
        s = off(x, short)
        m = off(product(s, s.t().contiguous()), short)
        p = b * m + c * product(m, m)
        d = p.diagonal().clone()
        p.diagonal().zero_()
        x = (a + d)[:, None] * x + product(off(p, short), s)
    return x.t() if g.shape[0] > g.shape[1] else x


def assert_near(got, g, dtype, scale=1.0, before=None, steps=5):
    want = exact(g, steps)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    off = max(float((noisy(g, dtype != BF16, gen, steps) - want).norm()) for _ in range(3)) * abs(scale)
    want = want * scale if before is None else want * scale + before.to(D)
    d = (got.to(D) - want).abs()
    step = HALF[dtype] * want.abs() + (2.0 ** -25 if dtype == F16 else 0.0)
    assert bool(torch.isfinite(got).all())
    assert float((d - step).clamp(min=0).norm()) <= 3 * off, (float(d.norm()), float(want.norm()), off)
    assert float((d - step).max()) <= 6 * 4.5 * off / want.numel() ** 0.5 + 1e-300


CASES = [
    (1, 1, 1, F32, F32, "normal", 0, 0), (1, 1, 64, F32, BF16, "normal", 0, 0), (1, 70, 1, BF16, F32, "normal", 3, 1), (2, 5, 7, F16, F16, "normal", 1, 0),
    (1, 64, 64, F32, F32, "gradient", 0, 0), (3, 33, 130, F32, BF16, "gradient", 1, 3), (2, 130, 33, BF16, F16, "gradient", 0, 1),
    (1, 127, 129, F32, F32, "few", 0, 0), (1, 128, 128, F16, BF16, "few", 8, 8), (2, 257, 300, F32, F32, "gradient", 0, 0),
    (5, 200, 333, F32, F32, "normal", 7, 0), (1, 1000, 512, BF16, BF16, "few", 0, 0), (3, 768, 768, F32, BF16, "gradient", 0, 0),
    (33, 72, 40, F32, F16, "normal", 0, 0), (2, 1536, 520, F32, F32, "few", 0, 0), (8, 1024, 1100, F32, BF16, "gradient", 0, 0),
    (1, 4100, 96, F32, F32, "gradient", 0, 0), (6, 1300, 1290, F32, F32, "gradient", 0, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}-{str(c[3])[6:]}-{str(c[4])[6:]}-{c[5]}")
def test_against_64_bits(case):
    print(case, flush=True)
    count, rows, cols, dtype, out_dtype, kind, pad, shift = case
    m = Make(rows + 3 * cols)
    given = [m.matrix(rows, cols, dtype, kind, pad, shift) for _ in range(count)]
    kept = [g.clone() for g in given]
    out = [torch.full((rows, cols + pad), 9.0, dtype=out_dtype, device=DEV)[:, :cols] for _ in range(count)]
    got = blocks.orthogonalise(given, out)
    assert got is not None and all(a is b for a, b in zip(got, out))
    for i in range(0, count, max(1, count // 3)):
        assert torch.equal(given[i], kept[i])
        assert_near(out[i], given[i], out_dtype)
    again = blocks.orthogonalise(given, [torch.empty(rows, cols, dtype=out_dtype, device=DEV) for _ in range(count)])
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    alone = blocks.orthogonalise(given[-1], torch.empty(rows, cols, dtype=out_dtype, device=DEV))
    assert float((alone.to(D) - out[-1].to(D)).norm()) <= 1e-2 * float(out[-1].to(D).norm())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows, cols", [(60, 100), (100, 60)])
def test_scaled_and_added(dtype, rows, cols):
    m = Make(4)
    g, before = m.matrix(rows, cols), m.normal(rows, cols).to(dtype)
    room = torch.zeros(rows, cols + 9, dtype=dtype, device=DEV)
    out = room[:, 2:2 + cols]
    out.copy_(before)
    blocks.orthogonalise(g, out, scale=-0.25, accumulate=True)
    assert_near(out, g, dtype, -0.25, before)
    assert bool((room[:, :2] == 0).all()) and bool((room[:, 2 + cols:] == 0).all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows, cols", [(1, 128), (128, 1), (31, 97), (64, 65), (65, 64), (128, 127), (128, 129), (129, 128), (16, 16)])
def test_small_sides(rows, cols, dtype):
    m = Make(rows + 5 * cols)
    g = m.matrix(rows, cols, dtype, "gradient", 3, 1)
    assert_near(blocks.orthogonalise(g), g, dtype)


def test_many_small_ones():      # more than a launch takes, some of them zeros or not finite
    m = Make(9)
    given = [m.matrix(20, 48) for _ in range(70)]
    given[5].zero_()
    given[40][3, 7] = float("inf")
    given[69][0, 0] = float("nan")
    kept = [g.clone() for g in given]
    out = blocks.orthogonalise(given, given)
    for i, g in enumerate(kept):
        if i in (40, 69):
            assert bool(out[i].isnan().all())
        elif i == 5:
            assert bool((out[i] == 0).all())
        else:
            assert_near(out[i], g, F32)


@pytest.mark.parametrize("steps", [1, 2, 3, 7])
def test_steps(steps):
    g = Make(5).matrix(96, 150)
    assert_near(blocks.orthogonalise(g, steps=steps), g, F32, steps=steps)


def test_over_the_updates_themselves():
    m = Make(6)
    for rows, cols in ((80, 200), (200, 80)):
        g = [m.matrix(rows, cols) for _ in range(3)]
        want = blocks.orthogonalise([v.clone() for v in g])
        blocks.orthogonalise(g, g)
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_singular_values():
    """Wide, tall and square: singular vectors stay, singular values lie near 1."""
    m = Make(7)
    for rows, cols in ((200, 300), (300, 200)):
        g = m.matrix(rows, cols)
        u, s, vh = torch.linalg.svd(g.to(D).cpu(), full_matrices=False)
        x = blocks.orthogonalise(g).to(D).cpu()
        inner = u.t() @ x @ vh.t()
        assert float((inner - torch.diag(inner.diagonal())).norm()) < 1e-3 * float(inner.norm())
        top = inner.diagonal()[s / s.norm() > 0.01]
        assert float(top.min()) > 0.6 and float(top.max()) < 1.3


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e10, 1e30])
def test_magnitudes(size):
    """Squares beyond fp32's range; below eps the result goes to zero with the update."""
    g = Make(8).matrix(50, 70) * size
    assert_near(blocks.orthogonalise(g), g, F32)
    if size >= 1e-12:
        assert_near(blocks.orthogonalise(g, eps=0.0), g * (1.0 / size), F32) if size >= 1 else None


@pytest.mark.parametrize("out", [F32, F16, BF16])
def test_zeros_and_what_is_not_finite(out):
    """Zeros stay zeros; an infinity or NaN leaves NaN, in its matrix alone."""
    m = Make(9)
    g = [m.matrix(40, 60), torch.zeros(40, 60, device=DEV), m.matrix(40, 60), m.matrix(40, 60)]
    want = blocks.orthogonalise(g[3], torch.empty(40, 60, dtype=out, device=DEV))
    g[0][3, 5] = float("nan")
    g[2][0, 0] = float("inf")
    got = blocks.orthogonalise(g, [torch.empty(40, 60, dtype=out, device=DEV) for _ in g])
    assert bool(got[0].isnan().all()) and bool((got[1] == 0).all()) and bool(got[2].isnan().all())
    assert torch.equal(got[3], want)
    rank_one = torch.outer(m.normal(40), m.normal(60))
    assert bool(torch.isfinite(blocks.orthogonalise(rank_one, torch.empty(40, 60, dtype=out, device=DEV))).all())


def test_slices_of_a_flat_buffer():
    """Matrices and results are slices of flat fp32 buffers, from odd elements on; what lies between stays."""
    m = Make(10)
    flat, to = m.normal(20_000), torch.full((20_000,), 4.0, device=DEV)
    cut = lambda f: [f[at:at + 48 * 56].view(48, 56) for at in (3, 3001, 9001)]  # noqa: E731
    blocks.orthogonalise(cut(flat), cut(to))
    for a, b in zip(cut(flat), cut(to)):
        assert_near(b, a, F32)
    mask = torch.ones(20_000, dtype=torch.bool, device=DEV)
    for v in cut(mask):
        v.fill_(False)
    assert bool((to[mask] == 4.0).all())


def test_another_stream_and_a_graph():
    m = Make(11)
    g = [m.matrix(150, 90) for _ in range(2)]
    eager = blocks.orthogonalise(g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = blocks.orthogonalise(g)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    out, graph = [torch.zeros(150, 90, device=DEV) for _ in g], torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        blocks.orthogonalise(g, out)
    first = [v.clone() for v in g]
    for replay in range(4):
        for o, v, f in zip(out, g, first):
            o.fill_(float("nan"))
            v.copy_(f if replay % 2 == 0 else f.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, blocks.orthogonalise(g))), replay
        assert torch.equal(out[0], eager[0]) == (replay % 2 == 0)
        assert float(torch.randn(1000, device=DEV).sum()) != 0.0


def test_one_workspace_and_what_it_held():
    m = Make(12)
    a, b = [m.matrix(100, 140) for _ in range(3)], m.matrix(300, 33)
    want = blocks.orthogonalise(a), blocks.orthogonalise(b)
    ws = torch.full((1 << 24,), 0xFF, dtype=torch.uint8, device=DEV)
    for _ in range(2):
        assert all(torch.equal(x, y) for x, y in zip(blocks.orthogonalise(a, workspace=ws), want[0]))
        assert torch.equal(blocks.orthogonalise(b, workspace=ws), want[1])
    with pytest.raises(dgs.DgsError) as err:
        blocks.orthogonalise(a, workspace=ws[:4096])
    assert err.value.code == dgs.DGS_ENOMEM


def test_refuses_what_is_elsewhere():
    g = torch.zeros(30, 20, device=DEV)
    for call in (lambda: blocks.orthogonalise(g.cpu()), lambda: blocks.orthogonalise([g, g.cpu()]), lambda: blocks.orthogonalise(g, g.cpu()),
                 lambda: blocks.orthogonalise(g, workspace=torch.zeros(1 << 20, dtype=torch.uint8))):
        with pytest.raises(dgs.DgsError) as err:
            call()
        assert err.value.code == dgs.DGS_EINVAL
