"""What the binding of the training blocks hands to the library, and what it remembers between two calls, without a GPU: on
host tensors, with the library's calls recorded in place of being made."""
import pytest

from paper_1910_10929_amd import blocks, dgs

torch = pytest.importorskip("torch")

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """The calls that the binding makes: the name and the packed arguments of each."""
    made = []
    monkeypatch.setattr(blocks, "_on_gpu", lambda t, what: t.get_device())
    monkeypatch.setattr(blocks, "_enqueue", lambda what, device, call, *args: made.append((what, args)))
    return made


def saved_of(rows, cols, **more):
    return blocks.Saved(rows, cols, device="cpu", **more)


@pytest.mark.parametrize("post", ["rms", None])
def test_values_kept_are_not_written_over(calls, post):
    """f is kept by reference for the backward pass: a u that lies over it is refused, unless a checkpoint is kept instead."""
    e = blocks.Edge(32, post=post, pre="layer")
    x, f = torch.zeros(6, 32), torch.zeros(6, 32, dtype=BF16)
    for u in (f, f.view(6, 32), f[:, :]):
        with pytest.raises(dgs.DgsError) as err:
            e.forward(x, f, u=u, save=saved_of(6, 32, checkpoints=False))
        assert err.value.code == dgs.DGS_EINVAL
    assert not calls
    same = torch.zeros(6, 32, dtype=BF16)
    for call in (lambda s: e.forward(same, f, x_out=f, save=s), lambda s: e.forward(x.bfloat16(), f, x_out=same, u=same, save=s),
                 lambda s: blocks.Edge(32, pre="layer").forward(same, u=same, save=s)):
        with pytest.raises(dgs.DgsError):
            call(saved_of(6, 32, checkpoints=False))
    assert not calls
    kept = saved_of(6, 32, checkpoints=False)
    e.forward(x, f, u=torch.empty_like(f), x_out=x, save=kept)
    assert kept.f is f and kept.x_out is x
    e.forward(x, f, u=f, save=saved_of(6, 32))
    e.forward(x, f, u=f)
    empty = torch.zeros(0, 32, dtype=BF16)      # (tensors without memory share no address)
    e.forward(torch.zeros(0, 32), empty, u=torch.zeros(0, 32, dtype=BF16), save=saved_of(0, 32, checkpoints=False))
    assert len(calls) == 4


def forward_of(args):
    """The packed arguments of a forward call, by name."""
    v = blocks._FORWARD.unpack(args[1])
    return dict(zip(("rows", "per", "stream", "type", "gate_type", "reserved", "x", "xs", "f", "fs", "gate", "gs", "xo", "xos", "u", "us", "pc", "pcs",
                     "pe", "pes", "nc", "ncs", "ne", "nes", "stats"), v))


def backward_of(args):
    v = blocks._BACKWARD.unpack(args[1])
    return dict(zip(("rows", "per", "stream", "type", "gate_type", "accumulate", "d", "ds", "du", "dus", "gate", "gs", "f", "fs", "x", "xs", "pc",
                     "pcs", "pe", "pes", "nc", "ncs", "ne", "nes", "stats", "dx", "dxs", "df", "dfs", "dg", "dgs", "gpw", "gpb", "gnw", "gnb", "ws",
                     "wsb"), v))


@pytest.mark.parametrize("coded", [True, False])
def test_an_edge_without_a_branch_stays_one(calls, coded):
    """What a Saved has room for says nothing about the forward pass: backward goes by what forward did, the last time."""
    first, inner = blocks.Edge(32, pre="layer"), blocks.Edge(32, post="rms", pre="layer")
    x, f = torch.zeros(6, 32), torch.zeros(6, 32)
    saved = saved_of(6, 32, checkpoints=coded)
    for branch in (False, True, False):
        e = inner if branch else first
        e.forward(x, f if branch else None, save=saved)
        assert (forward_of(calls[-1][1])["pc"] != 0) == (branch and coded)
        dx, df = e.backward(saved, dx_out=x, du=f)
        a = backward_of(calls[-1][1])
        assert (df is not None) == branch and (a["df"] != 0) == branch
        assert (a["pc"] != 0) == (branch and coded) and (a["f"] != 0) == (branch and not coded)
        assert (a["nc"] != 0) == coded and (a["x"] != 0) == (not coded)
        if not branch:
            with pytest.raises(dgs.DgsError):
                e.backward(saved, dx_out=x, du=f, df=torch.zeros(6, 32))


def test_saved_that_is_put_together_by_hand(calls):
    """Without a forward pass, what it holds says what the edge has."""
    c = lambda: blocks.Checkpoint(6, 32, "cpu")  # noqa: E731
    x = torch.zeros(6, 32)
    e, first = blocks.Edge(32, post="rms", pre="layer"), blocks.Edge(32, pre="layer")
    assert e.backward(saved_of(6, 32, post=c(), pre=c()), dx_out=x, du=x)[1] is not None
    assert e.backward(saved_of(6, 32, f=x.clone(), x_out=x), dx_out=x, du=x)[1] is not None
    assert first.backward(saved_of(6, 32, pre=c()), dx_out=x, du=x)[1] is None
    # what a forward pass with a branch kept has been taken away
    saved = saved_of(6, 32)
    e.forward(x, x.clone(), save=saved)
    saved.post = None
    with pytest.raises(dgs.DgsError):
        e.backward(saved, dx_out=x, du=x)


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("stream, kind", [(F32, BF16), (F32, F16), (F32, F32), (BF16, BF16)])
def test_gradients_have_the_types_of_the_forward_pass(calls, stream, kind, coded):
    """Where a gradient is absent and no place is given for the result, its type is that of x or f -- not the other one's."""
    e, last, first = blocks.Edge(32, post="rms", pre="layer"), blocks.Edge(32, post="rms"), blocks.Edge(32, pre="rms")
    x, f = torch.zeros(6, 32, dtype=stream), torch.zeros(6, 32, dtype=kind)
    gate = torch.zeros(1, 32, dtype=kind)
    number = lambda t: blocks._TYPES[t]  # noqa: E731
    saved = saved_of(6, 32, checkpoints=coded)
    e.forward(x, f, gate=gate, save=saved)
    dx, df = e.backward(saved, du=f, gate=gate)
    assert (dx.dtype, df.dtype) == (stream, kind)
    last.forward(x, f, gate=gate, save=saved)
    dx, df = last.backward(saved, dx_out=x, gate=gate, dgate=torch.zeros_like(gate))
    assert (dx.dtype, df.dtype) == (stream, kind)
    a = backward_of(calls[-1][1])
    assert (a["stream"], a["type"], a["gate_type"]) == (number(stream), number(kind), number(kind))
    first.forward(x, u=torch.zeros(6, 32, dtype=kind), save=saved)
    dx, df = first.backward(saved, du=f)
    assert dx.dtype == stream and df is None


def test_gradients_of_other_types_than_the_forward_pass(calls):
    """What is given goes before what was remembered, and what was remembered is left where it does not go with that."""
    e = blocks.Edge(32, post="rms", pre="layer")
    half, full = torch.zeros(6, 32, dtype=BF16), torch.zeros(6, 32)
    saved = saved_of(6, 32)
    e.forward(half, half.clone(), save=saved)
    assert [t.dtype for t in e.backward(saved, dx_out=full, du=full)] == [F32, F32]
    assert [t.dtype for t in e.backward(saved, du=full)] == [F32, F32]
    assert [t.dtype for t in e.backward(saved, du=half, dx=full)] == [F32, BF16]
    assert [t.dtype for t in e.backward(saved, dx_out=full)] == [F32, BF16]
    assert [t.dtype for t in e.backward(saved, dx_out=full, df=full)] == [F32, F32]
    # nothing remembered: as the gradient that is there
    by_hand = saved_of(6, 32, stats=saved.stats, post=saved.post, pre=saved.pre)
    assert [t.dtype for t in e.backward(by_hand, du=half)] == [BF16, BF16]
    assert [t.dtype for t in e.backward(by_hand, dx_out=full)] == [F32, F32]


@pytest.mark.parametrize("gates, per", [(0, None), (0, 5), (1, None), (1, 7), (3, None), (3, 2)])
def test_no_rows_under_a_gate(calls, gates, per):
    """A batch without rows takes the gate that other batches take; its gradient is zero, or with accumulate what it was."""
    e = blocks.Edge(32, post="rms", pre="layer")
    none = torch.zeros(0, 32)
    saved = saved_of(0, 32)
    for kind in (F32, BF16):
        f = none.to(kind)
        gate = torch.zeros(gates, 32, dtype=kind)
        xo, u = e.forward(none, f, gate=gate, rows_per_gate=per, save=saved)
        assert xo.shape == u.shape == (0, 32)
        for accumulate in (False, True):
            dgate = torch.full_like(gate, 3.0)
            e.backward(saved, dx_out=none, du=f, gate=gate, rows_per_gate=per, dgate=dgate, accumulate=accumulate)
            assert bool((dgate == (3.0 if accumulate and kind == F32 else 0.0)).all())
    assert len(calls) == 6
    for bad in (dict(gate=torch.zeros(1, 31)), dict(gate=torch.zeros(32)), dict(gate=torch.zeros(1, 32), rows_per_gate=0)):
        with pytest.raises(dgs.DgsError):
            e.forward(none, none, **bad)


def large(rows, cols, dtype):
    """A matrix without memory."""
    return torch.empty(rows, cols, dtype=dtype, device="meta")


@pytest.mark.parametrize("rows, cols", [(2 ** 31, 1), (2 ** 32, 1), (2 ** 32 + 5, 3), (1, 2 ** 32), (2, 2 ** 32 + 64)])
def test_sizes_beyond_32_bits(calls, rows, cols):
    """Sizes go to the library in 32 bits: what does not fit is refused, and not taken for what is left of it."""
    x = large(rows, cols, F32)
    bad = [
        lambda: blocks.Checkpoint(rows, cols, "meta"), lambda: blocks.Checkpoint.of(large(rows, cols, torch.int8), large(rows, (cols + 31) // 32, torch.uint8)),
        lambda: blocks.Saved(rows, cols, "meta"), lambda: blocks.Edge(cols, pre="rms").forward(x), lambda: blocks.Edge(cols, post="rms").forward(x, x),
        lambda: blocks.Edge(cols, post="rms").backward(blocks.Saved(rows, cols, "meta", checkpoints=False, f=x), dx_out=x),
        lambda: blocks.weight_grad(large(4, max(rows, cols), F32), blocks.Checkpoint(4, 32, "meta"), large(max(rows, cols), 32, F32)),
    ]
    for call in bad:
        with pytest.raises(dgs.DgsError) as err:
            call()
        assert err.value.code == dgs.DGS_ENOTSUP
    assert not calls


def test_more_rows_for_a_gate_row_than_there_are(calls):
    x = torch.zeros(6, 32)
    blocks.Edge(32, post="rms").forward(x, x.clone(), gate=x[:1], rows_per_gate=2 ** 40)
    assert forward_of(calls[0][1])["per"] >= 6


def test_what_is_no_matrix(calls):
    m, c = torch.zeros(6, 32), blocks.Checkpoint(6, 32, "cpu")
    e, saved = blocks.Edge(32, post="rms", pre="layer"), saved_of(6, 32)
    for wrong in (torch.zeros(()), torch.zeros(32), torch.zeros(1, 6, 32)):
        for call in (lambda: blocks.Checkpoint.of(wrong.to(torch.int8), c.exps), lambda: blocks.Checkpoint.of(c.codes, wrong.to(torch.uint8)),
                     lambda: c.encode(wrong), lambda: c.decode(out=wrong), lambda: e.forward(wrong, m), lambda: e.forward(m, wrong),
                     lambda: e.forward(m, m, gate=wrong), lambda: e.forward(m, m, gate=wrong, rows_per_gate=6),
                     lambda: e.backward(saved, dx_out=wrong, du=m), lambda: e.backward(saved, dx_out=m, du=m, gate=m[:1], dgate=wrong),
                     lambda: blocks.weight_grad(wrong, c, m), lambda: blocks.weight_grad(m, c, wrong)):
            with pytest.raises(dgs.DgsError) as err:
                call()
            assert err.value.code == dgs.DGS_EINVAL
    assert not calls
