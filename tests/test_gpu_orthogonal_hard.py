"""Orthogonalised updates (blocks.orthogonalise) where numbers are hard: coefficients that take little or nothing off small singular
values, against the same steps in 64 bits, on both paths (a launch for all steps up to 128 x 128, launches a step beyond).

Tolerances.  A step rounds X by 2^-21 (bfloat16 results: 2^-10) for the operands, by 2^-24 sqrt(n) for a sum of n products (three pairs of
parts, to either side), and by 2^-37 of 1, since X's smallest values have fewer bits.  What a step leaves grows as the map's slopes say: by 2 a
step at the fixed point 1 of (0.5, 0.5, 0); relative to X by less than 2 in all on the way to 0 of (0.75, 0.5, -0.25) from singular values of
0.42 and less; (1, 0.9, -0.9) takes what the steps to 1 leave off again (slope -0.8 there)."""
import pytest

from paper_1910_10929_amd import blocks, dgs

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"
F32, F16, BF16, D = torch.float32, torch.float16, torch.bfloat16, torch.float64
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def built():
    assert torch.cuda.is_available()
    dgs.lib()


def matrix(rows, cols, norm, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + rows + 3 * cols)
    m = torch.randn(rows, cols, device=DEV, generator=g)
    return m * (norm / m.norm())


def steps64(g, steps, coefficients, eps):
    a, b, c = (torch.tensor(v, dtype=F32).to(D).item() for v in coefficients)
    x = g.to(D)
    x = x / (torch.linalg.vector_norm(x) + torch.tensor(eps, dtype=F32).to(D).item())
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for _ in range(steps):
        m = x @ x.t()
        x = a * x + (b * m + c * (m @ m)) @ x
    return x.t() if tall else x


def assert_near(got, want, grown, steps):
    d = (got.to(D) - want).abs() - HALF[got.dtype] * want.abs() - (2.0 ** -25 if got.dtype == F16 else 0.0)
    assert bool(torch.isfinite(got).all())
    off = (2.0 ** -10 if got.dtype == BF16 else 2.0 ** -21) + 2.0 ** -24 * (3.0 * max(want.shape)) ** 0.5
    assert float(d.clamp(min=0).norm()) <= float(want.norm()) * grown * off + steps * 2.0 ** -37 * want.numel() ** 0.5


# rows, columns, coefficients, steps, norm, eps, what a step's error grows to
COEFFICIENTS = [
    (1, 1, (0.5, 0.5, 0.0), 7, 1.0, 1e-7, 127), (1, 200, (0.5, 0.5, 0.0), 10, 1.0, 1e-7, 1023), (300, 1, (0.5, 0.5, 0.0), 10, 1.0, 1e-7, 1023),
    (20, 30, (0.75, 0.5, -0.25), 40, 1.0, 1e-7, 80), (9, 140, (0.75, 0.5, -0.25), 40, 1.0, 1e-7, 80), (700, 300, (0.75, 0.5, -0.25), 40, 1.0, 1e-7, 80),
    (1, 40, (1.0, 0.9, -0.9), 180, 0.0661, 1.0, 180), (130, 1, (1.0, 0.9, -0.9), 180, 0.0661, 1.0, 180),
    (9, 20, (0.25, 0.5, 0.25), 5, 1e-5, 1.0, 5), (140, 30, (0.25, 0.5, 0.25), 5, 1e-5, 1.0, 5),
]


@pytest.mark.parametrize("out", [F32, F16, BF16])
@pytest.mark.parametrize("case", COEFFICIENTS, ids=lambda c: f"{c[0]}x{c[1]}-{c[2]}")
def test_coefficients(case, out):
    print(case, out, flush=True)
    rows, cols, coefficients, steps, norm, eps, grown = case
    g = matrix(rows, cols, norm)
    got = blocks.orthogonalise(g, torch.empty(rows, cols, dtype=out, device=DEV), steps=steps, coefficients=coefficients, eps=eps)
    assert_near(got, steps64(g, steps, coefficients, eps), grown, steps)
