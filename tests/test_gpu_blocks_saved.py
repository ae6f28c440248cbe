"""What an edge's forward pass leaves in a `Saved` and its backward pass takes from there, against plain computations in 64
bits; tolerances as in test_gpu_blocks."""
import pytest

from paper_1910_10929_amd import blocks, dgs

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_blocks import BF16, D, DEV, EPS, F16, F32, Case, assert_near, backward64, run_backward, values64  # noqa: E402

# rows, cols, stream, type, post, pre, biases, rows for each gate row, gate type, padding
FIRST = [
    (1, 768, F32, F32, None, "rms", True, 0, F32, 0),
    (67, 7, F16, F16, None, "layer", True, 0, F32, 1),
    (300, 768, F32, F32, None, "layer", True, 0, F32, 0),
    (130, 1001, BF16, BF16, None, "rms", False, 0, F32, 3),
    (5, 9000, F32, F32, None, "layer", True, 0, F32, 0),
]


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("case", FIRST, ids=lambda c: f"{c[0]}x{c[1]}")
def test_backward_without_a_branch(case, coded):
    """The first edge of a model, with a Saved that has room for a branch and held one in the step before."""
    c = Case(case, seed=3, branch=False)
    rows, cols = c.rows, c.cols
    saved = blocks.Saved(rows, cols, device=DEV, checkpoints=coded)
    other = Case(case, seed=4)
    other.edge.forward(other.x, other.f, save=saved)
    c.edge.forward(c.x, save=saved)
    d_in, u_in = c.make(rows, cols, c.stream, c.pad, shift=1), c.make(rows, cols, c.type, c.pad)
    stats = saved.stats.to(D)
    xh = values64(saved.pre) if coded else (c.x.to(D) - stats[:, 2:3]) * stats[:, 3:4]
    want = backward64(c, d_in, u_in, None, xh, stats)
    got = run_backward(c, saved, d_in, u_in)
    assert "df" not in got
    size = c.skip * (d_in.to(D).abs().amax(1, keepdim=True) + stats[:, 3:4] * (u_in.to(D) * c.w("pre_weight", 1.0)).abs().amax(1, keepdim=True)
                     * (1 + xh.abs().amax(1, keepdim=True).square()))
    assert_near(got["dx"], want["dx"], size, "dx")
    for name in ("pre_weight", "pre_bias"):
        terms = want["size_" + name]
        assert_near(got[name], want[name], terms.abs().amax(0), name, extra=8 * rows ** 0.5 * EPS * terms.square().sum(0).sqrt())
    with pytest.raises(dgs.DgsError):
        c.edge.backward(saved, dx_out=d_in, du=u_in, post_weight_grad=torch.zeros(cols, device=DEV))


@pytest.mark.parametrize("coded", [True, False])
def test_absent_gradients_without_places_for_the_results(coded):
    """An fp32 stream with a bfloat16 branch: a gradient that is absent is one of zeros, and changes no result's type."""
    c = Case((50, 96, F32, BF16, "rms", "layer", True, 7, BF16, 0))
    saved = blocks.Saved(50, 96, device=DEV, checkpoints=coded)
    c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=7, save=saved)
    d, u = c.make(50, 96, F32), c.make(50, 96, BF16)
    for have, zeros in ((dict(d_in=d, u_in=None), dict(d_in=d, u_in=torch.zeros_like(u))), (dict(d_in=None, u_in=u), dict(d_in=torch.zeros_like(d), u_in=u))):
        a, b = run_backward(c, saved, **have), run_backward(c, saved, **zeros)
        assert (a["dx"].dtype, a["df"].dtype) == (F32, BF16)
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_no_rows_under_a_gate():
    e = blocks.Edge(64, post="rms", pre="layer")
    x = torch.empty(0, 64, device=DEV)
    gate = torch.ones(1, 64, device=DEV)
    saved = blocks.Saved(0, 64, device=DEV)
    xo, u = e.forward(x, x.clone(), gate=gate, save=saved)
    assert xo.shape == u.shape == (0, 64)
    dgate, grad = torch.full((1, 64), 3.0, device=DEV), torch.full((64,), 3.0, device=DEV)
    e.backward(saved, dx_out=x, du=x, gate=gate, dgate=dgate, post_weight_grad=grad, accumulate=True)
    assert bool((dgate == 3.0).all()) and bool((grad == 3.0).all())
    e.backward(saved, dx_out=x, du=x, gate=gate, dgate=dgate, post_weight_grad=grad)
    assert bool((dgate == 0.0).all()) and bool((grad == 0.0).all())
