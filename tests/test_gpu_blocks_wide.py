"""Edges of rows that take twelve or sixteen wavefronts, with more rows than there are workgroups: every one goes round two or
three times, the last ones fewer.  The comparisons and their tolerances are those of test_gpu_blocks."""
import pytest

from paper_1910_10929_amd import blocks

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import test_gpu_blocks as base  # noqa: E402
from test_gpu_blocks import BF16, D, DEV, EPS, F16, F32, Case, assert_near, backward64, gates64, run_backward, values64  # noqa: E402

# rows, cols, stream, type, post, pre, biases, rows for each gate row, gate type, padding: no gate, one gate row, several with
# rows in parts, and one to a few rows, whole ones of which go to a workgroup
WIDE = [
    (611, 6000, F32, BF16, "layer", "layer", True, 0, F32, 1),
    (611, 6000, F16, F16, "rms", "layer", True, 1, F16, 0),
    (611, 5001, BF16, BF16, "layer", "rms", True, 250, BF16, 3),
    (611, 8192, BF16, BF16, "rms", "rms", True, 611, F32, 0),
    (611, 8192, F32, F32, "layer", "rms", True, 2, F32, 0),
    (611, 7003, F32, F16, "rms", "layer", True, 0, F32, 0),
    (611, 10001, BF16, BF16, "layer", "layer", True, 2, BF16, 1),
    (611, 10001, F32, F32, "rms", "layer", True, 611, F32, 0),
    (611, 12000, F16, F16, "layer", "rms", True, 250, F32, 0),
    (300, 16384, F32, BF16, "layer", "layer", True, 0, F32, 0),
]


@pytest.mark.parametrize("case", WIDE, ids=lambda c: f"{c[0]}x{c[1]}")
def test_forward(case):
    base.test_edge_forward(case, True)


@pytest.mark.parametrize("case", WIDE[::4], ids=lambda c: f"{c[0]}x{c[1]}")
def test_forward_without_a_branch(case):
    base.test_edge_forward(case, False)


@pytest.mark.parametrize("case", WIDE, ids=lambda c: f"{c[0]}x{c[1]}")
def test_backward(case):
    """From checkpoints: normalised values that are exact, as the tolerance of the gates' gradients wants them."""
    base.test_edge_backward(case, True)


def pieces(c, most=200):
    """The rows in runs so short that every workgroup has one row at most, with the gate of each and its rows for a gate row."""
    step = c.per if c.per > most else most // (c.per or 1) * (c.per or 1)
    for lo in range(0, c.rows, step):
        hi = min(lo + step, c.rows)
        if c.per <= most:
            yield slice(lo, hi), None if c.gate is None else c.gate[lo // c.per:(hi + c.per - 1) // c.per], c.per or None
        else:
            for at in range(lo, hi, most):
                yield slice(at, min(at + most, hi)), c.gate[lo // c.per:lo // c.per + 1], c.per


def part_of(saved, rows, x_out):
    """What was saved of some rows."""
    n = rows.stop - rows.start
    cut = lambda k: None if k is None else blocks.Checkpoint.of(k.codes[rows], k.exps[rows])  # noqa: E731
    if saved.post is None:
        return blocks.Saved(n, saved.cols, stats=saved.stats[rows], f=saved.f[rows], x_out=x_out[rows])
    return blocks.Saved(n, saved.cols, stats=saved.stats[rows], post=cut(saved.post), pre=cut(saved.pre))


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("case", WIDE, ids=lambda c: f"{c[0]}x{c[1]}")
def test_a_row_is_the_same_in_any_round(case, coded):
    """What a row gives does not depend on which round of its workgroup it comes in: the same bits as in calls of few rows, and
    so does the gradient of a gate row that one team has to itself.  Sums over rows against 64 bits."""
    c = Case(case, seed=7)
    rows, cols = c.rows, c.cols
    saved = blocks.Saved(rows, cols, device=DEV, checkpoints=coded)
    xo, u = c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=c.per or None, save=saved)
    d, du = c.make(rows, cols, c.stream, c.pad), c.make(rows, cols, c.type, c.pad)
    got = run_backward(c, saved, d, du, start=float("nan"))
    for part, gate, per in pieces(c):
        n = part.stop - part.start
        few = blocks.Saved(n, cols, device=DEV, checkpoints=coded)
        x2, u2 = c.edge.forward(c.x[part], c.f[part], gate=gate, rows_per_gate=per, save=few)
        assert torch.equal(x2, xo[part]) and torch.equal(u2, u[part]) and torch.equal(few.stats, saved.stats[part])
        if coded:
            for a, b in ((few.post, saved.post), (few.pre, saved.pre)):
                assert torch.equal(a.codes, b.codes[part]) and torch.equal(a.exps, b.exps[part])
        dgate = None if gate is None else torch.empty_like(gate)
        dx, df = c.edge.backward(part_of(saved, part, xo), dx_out=d[part], du=du[part], gate=gate, rows_per_gate=per, dgate=dgate)
        assert torch.equal(dx, got["dx"][part]) and torch.equal(df, got["df"][part])
        if c.per == 1:
            assert torch.equal(dgate, got["dgate"][part])
    stats = saved.stats.to(D)
    if coded:
        fh, xh = values64(saved.post), values64(saved.pre)
    else:
        fh, xh = (c.f.to(D) - stats[:, 0:1]) * stats[:, 1:2], (xo.to(D) - stats[:, 2:3]) * stats[:, 3:4]
    want = backward64(c, d, du, fh, xh, stats)
    top = d.to(D).abs().amax(1, keepdim=True) + (stats[:, 3:4] * (du.to(D) * c.w("pre_weight", 1.0)).abs().amax(1, keepdim=True)
                                                 * (1 + xh.abs().amax(1, keepdim=True).square()))
    top_m = top * c.branch * (gates64(c.gate, c.per, rows).abs().amax(1, keepdim=True) if c.gate is not None else 1.0)
    for name in ("post_weight", "post_bias", "pre_weight", "pre_bias"):
        terms = want["size_" + name]
        # each term of a post gradient is off by what its row's d is off by; of a pre gradient's weight, by its own rounding
        err_in = (top_m if name.startswith("post") else top * 0) * (fh.abs() if name == "post_weight" else 1.0)
        assert_near(got[name], want[name], terms.abs().amax(0), name,
                    extra=8 * rows ** 0.5 * EPS * terms.square().sum(0).sqrt() + 64 * EPS * err_in.square().sum(0).sqrt())


@pytest.mark.parametrize("case", [WIDE[1], WIDE[4], WIDE[6], WIDE[8]], ids=lambda c: f"{c[0]}x{c[1]}")
def test_in_place_and_repeatable(case):
    c = Case(case)
    saved, saved2 = blocks.Saved(c.rows, c.cols, device=DEV), blocks.Saved(c.rows, c.cols, device=DEV)
    xo, u = c.edge.forward(c.x, c.f, gate=c.gate, rows_per_gate=c.per or None, save=saved)
    x2, f2 = c.x.clone(), c.f.clone()
    c.edge.forward(x2, f2, gate=c.gate, rows_per_gate=c.per or None, x_out=x2, u=f2, save=saved2)
    assert torch.equal(xo, x2) and torch.equal(u, f2)
    for a, b in ((saved.post, saved2.post), (saved.pre, saved2.pre)):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.exps, b.exps)
    d, du = c.make(c.rows, c.cols, c.stream), c.make(c.rows, c.cols, c.type)
    one, two = run_backward(c, saved, d, du), run_backward(c, saved, d, du)
    d2, du2 = d.clone(), du.clone()
    three = run_backward(c, saved, d2, du2, dx=d2, df=du2)
    for k in one:
        assert torch.equal(one[k], two[k]) and torch.equal(one[k], three[k]), k
