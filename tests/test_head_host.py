"""Host side of the output layer and of orthogonalised updates, without a GPU: what the C ABI refuses -- all of it before anything
is enqueued -- workspace sizes, and what the binding hands to the library."""
import ctypes
import struct

import pytest

from paper_1910_10929_amd import blocks, dgs

torch = pytest.importorskip("torch")

EINVAL, ENOMEM, ENOTSUP = dgs.DGS_EINVAL, dgs.DGS_ENOMEM, dgs.DGS_ENOTSUP
P = 1 << 20      # a pointer that is never followed
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16

HEAD = dict(rows=4, cols=96, vocab=100, type=2, target=8, accumulate=0, x=P, xs=96, w=P, ws=96, bias=0, targets=P, loss=P, lse=P, dloss=0,
            dlse=0, dx=P, dxs=96, dw=P, dws=96, db=P, work=P, bytes=1 << 40)


def head(call, **change):
    a = dict(HEAD, **change)
    assert set(change) <= set(HEAD)
    return getattr(blocks.lib(), call)(blocks._HEAD.pack(*a.values()), None)


BOTH = [
    (EINVAL, dict(cols=0)), (EINVAL, dict(vocab=0)), (EINVAL, dict(type=3)), (EINVAL, dict(target=2)),
    (EINVAL, dict(x=0)), (EINVAL, dict(x=P + 1)), (EINVAL, dict(xs=95)), (EINVAL, dict(w=0)), (EINVAL, dict(ws=95)), (EINVAL, dict(w=P + 1)),
    (EINVAL, dict(bias=P + 2)), (EINVAL, dict(targets=0)), (EINVAL, dict(targets=P + 4)), (EINVAL, dict(lse=0)), (EINVAL, dict(lse=P + 1)),
    (EINVAL, dict(work=0)), (EINVAL, dict(work=P + 8)), (ENOMEM, dict(bytes=100)),
    (ENOTSUP, dict(cols=(1 << 20) + 8, xs=1 << 21, ws=1 << 21, dxs=1 << 21, dws=1 << 21)), (EINVAL, dict(xs=1 << 32)), (EINVAL, dict(ws=1 << 32)),
    (ENOTSUP, dict(rows=(1 << 24) + 1)), (ENOTSUP, dict(vocab=(1 << 24) + 1)),
    (ENOTSUP, dict(rows=1 << 20, vocab=(1 << 18) + 1)), (ENOTSUP, dict(rows=1 << 24, cols=1032, xs=1032, ws=1032, dxs=1032, dws=1032)),
]


@pytest.mark.parametrize("code, change", BOTH + [(EINVAL, dict(loss=P + 2))])
def test_forward_refuses(code, change):
    assert head("dgs_head_forward", **change) == code


@pytest.mark.parametrize("code, change", BOTH + [
    (EINVAL, dict(dx=P + 1)), (EINVAL, dict(dxs=95)), (EINVAL, dict(dw=P + 2)), (EINVAL, dict(dws=95)), (EINVAL, dict(db=P + 1)),
    (EINVAL, dict(dloss=P + 1)), (EINVAL, dict(dlse=P + 2)),
])
def test_backward_refuses(code, change):
    assert head("dgs_head_backward", **change) == code


def test_null_structures_and_nothing_to_do():
    L = blocks.lib()
    assert L.dgs_head_forward(None, None) == EINVAL and L.dgs_head_backward(None, None) == EINVAL and L.dgs_orthogonalise(None, None) == EINVAL
    assert L.dgs_head_workspace(None, 0) == 0 and L.dgs_orthogonalise_workspace(None) == 0
    assert head("dgs_head_forward", rows=0, x=0, targets=0, lse=0, work=0, bytes=0) == 0
    assert head("dgs_head_backward", rows=0, x=0, targets=0, lse=0, dw=0, db=0) == 0
    assert ortho(count=0) == 0


def test_workspace_sizes():
    def need(backward, **change):
        return blocks.lib().dgs_head_workspace(blocks._HEAD.pack(*dict(HEAD, **change).values()), backward)
    assert need(0, cols=0) == 0 and need(1, type=5) == 0
    big = dict(rows=8192, cols=768, vocab=30522, xs=768, ws=768, dxs=768, dws=768)
    # no logits: a maximum and a sum for each tile's rows; in the backward pass a piece of the logits' gradient and copies
    assert need(0, **big) < 8192 * 30522 // 8
    assert need(1, **big) < (1 << 30) + (1 << 29)
    assert need(1, **dict(big, rows=1 << 20, vocab=1 << 17)) < (1 << 33) + (1 << 28) + (1 << 20) * 768 * 16
    # a matrix that is not laid out in pieces of sixteen bytes is copied
    assert need(0, **dict(big, w=P + 2)) >= need(0, **big) + 30522 * 768 * 2
    assert need(0, **dict(big, ws=769)) == need(0, **dict(big, w=P + 2)) == need(0, **dict(big, ws=1 << 21))
    assert need(0, **dict(big, xs=1 << 31)) >= need(0, **big) + 8192 * 768 * 2
    assert need(0, **dict(big, rows=1, xs=1 << 31)) == need(0, **dict(big, rows=1))


ORTHO = dict(count=2, rows=40, cols=50, steps=5, type=0, out=0, accumulate=0, reserved=0, a=3.4, b=-4.8, c=2.0, eps=1e-7, scale=1.0,
             inp=None, outp=None, work=P, bytes=1 << 40)


def ortho(places=None, out_places=None, call="dgs_orthogonalise", **change):
    table = ctypes.create_string_buffer(struct.pack("@8Q", *(places or (P, 50, P, 50)), *(out_places or (P, 50, P, 50))))
    at = ctypes.addressof(table)
    a = dict(ORTHO, inp=at, outp=at + 32)
    assert set(change) <= set(a)
    a.update(change)
    packed = blocks._ORTHOGONALISE.pack(*a.values())
    return blocks.lib().dgs_orthogonalise(packed, None) if call == "dgs_orthogonalise" else blocks.lib().dgs_orthogonalise_workspace(packed)


@pytest.mark.parametrize("code, change", [
    (EINVAL, dict(rows=0)), (EINVAL, dict(cols=0)), (EINVAL, dict(steps=0)), (EINVAL, dict(type=3)), (EINVAL, dict(out=-1)),
    (EINVAL, dict(eps=-1.0)), (EINVAL, dict(eps=float("nan"))), (EINVAL, dict(inp=0)), (EINVAL, dict(outp=0)),
    (EINVAL, dict(places=(P, 50, 0, 50))), (EINVAL, dict(places=(P, 49, P, 50))), (EINVAL, dict(places=(P + 2, 50, P, 50))),
    (EINVAL, dict(out_places=(P, 50, P, 1 << 32))), (EINVAL, dict(out_places=(P, 50, P + 1, 50))),
    (EINVAL, dict(work=0)), (EINVAL, dict(work=P + 8)), (ENOMEM, dict(bytes=1000)),
    (ENOTSUP, dict(rows=65537)), (ENOTSUP, dict(cols=65537)),
])
def test_orthogonalise_refuses(code, change):
    assert ortho(**change) == code


def test_orthogonalise_workspace():
    need = lambda **k: ortho(call="workspace", **k)  # noqa: E731
    assert need(steps=0) == 0 and need(count=0) == 0
    # X twice and two squares, in two halves where the result is fp32 or half
    assert need(count=1, rows=512, cols=1024, out=2) >= 2 * (2 * 512 * 1024 * 2) + 2 * 512 * 512 * 2
    assert need(count=1, rows=512, cols=1024) >= need(count=1, rows=512, cols=1024, out=2) + 2 * 512 * 512 * 2
    assert need(count=1000, rows=512, cols=1024) == need(count=32, rows=512, cols=1024)


# -- the binding ----------------------------------------------------------------------

@pytest.fixture
def calls(monkeypatch):
    """The calls that the binding makes: the name and the packed arguments of each."""
    made = []
    monkeypatch.setattr(blocks, "_on_gpu", lambda t, what: t.get_device())
    monkeypatch.setattr(blocks, "_enqueue", lambda what, device, call, *args: made.append((what, args)))
    return made


def head_of(args):
    return dict(zip(HEAD, blocks._HEAD.unpack(args[0])))


def test_head_hands_over(calls):
    w, bias = torch.zeros(50, 40, dtype=BF16), torch.zeros(50)
    h = blocks.Head(w, bias)
    x, t = torch.zeros(6, 48, dtype=BF16)[:, :40], torch.zeros(6, dtype=torch.int32)
    loss, lse = h.forward(x, t)
    assert loss.shape == lse.shape == (6,) and loss.dtype == lse.dtype == F32
    a = head_of(calls[0][1])
    assert (a["rows"], a["cols"], a["vocab"], a["type"], a["target"]) == (6, 40, 50, 2, 4)
    assert (a["x"], a["xs"], a["w"], a["ws"], a["bias"]) == (x.data_ptr(), 48, w.data_ptr(), 40, bias.data_ptr())
    assert (a["loss"], a["lse"], a["dx"], a["dw"]) == (loss.data_ptr(), lse.data_ptr(), 0, 0)
    dw = torch.zeros(50, 44)[:, :40]
    dx = h.backward(x, t.long(), lse, dloss=loss, dweight=dw, accumulate=True)
    b = head_of(calls[1][1])
    assert dx.shape == (6, 40) and dx.dtype == BF16
    assert (b["dx"], b["dxs"], b["dw"], b["dws"], b["db"], b["dloss"], b["dlse"]) == (dx.data_ptr(), 40, dw.data_ptr(), 44, 0, loss.data_ptr(), 0)
    assert (b["target"], b["accumulate"]) == (8, 1)
    assert h.backward(x, t, lse, dweight=dw, need_dx=False) is None and head_of(calls[2][1])["dx"] == 0


def test_head_refuses(calls):
    w = torch.zeros(50, 40)
    h, x, t, v = blocks.Head(w), torch.zeros(6, 40), torch.zeros(6, dtype=torch.int64), torch.zeros(6)
    bad = [
        lambda: blocks.Head(w[0]), lambda: blocks.Head(w.double()), lambda: blocks.Head(w, torch.zeros(40)), lambda: blocks.Head(w.t()),
        lambda: blocks.Head(w[:0]), lambda: blocks.Head(w[:, :0]), lambda: blocks.Head(w, torch.zeros(50, dtype=BF16)),
        lambda: h.forward(x[0], t), lambda: h.forward(x[:, :39], t), lambda: h.forward(x.bfloat16(), t), lambda: h.forward(x, t[:5]),
        lambda: h.forward(x, t.float()), lambda: h.forward(x, torch.zeros(12, dtype=torch.int64)[::2]), lambda: h.forward(x, t, loss=v[:5]),
        lambda: h.forward(x, t, lse=v.double()), lambda: h.forward(x.t().contiguous().t(), t),
        lambda: h.backward(x, t, None), lambda: h.backward(x, t, v[:3]), lambda: h.backward(x, t, v, dloss=v.half()),
        lambda: h.backward(x, t, v, dlse=v[:1]), lambda: h.backward(x, t, v, dx=x.bfloat16()), lambda: h.backward(x, t, v, dx=torch.zeros(5, 40)),
        lambda: h.backward(x, t, v, dx=torch.zeros(6, 40), need_dx=False), lambda: h.backward(x, t, v, dx=x),
        lambda: h.backward(x, t, v, dweight=w.bfloat16()), lambda: h.backward(x, t, v, dweight=w[:40]), lambda: h.backward(x, t, v, dbias=v),
        lambda: h.backward(x, t, v, dweight=w),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(dgs.DgsError) as err:
            call()
        assert err.value.code == EINVAL, i
    assert not calls


def test_orthogonalise_hands_over(calls):
    g = [torch.zeros(30, 20) for _ in range(3)]
    out = blocks.orthogonalise(g, scale=0.5)
    assert len(out) == 3 and all(o.shape == (30, 20) and o.dtype == F32 for o in out)
    a = dict(zip(ORTHO, blocks._ORTHOGONALISE.unpack(calls[0][1][0])))
    assert (a["count"], a["rows"], a["cols"], a["steps"], a["type"], a["out"], a["accumulate"], a["scale"]) == (3, 30, 20, 5, 0, 0, 0, 0.5)
    same = blocks.orthogonalise(g[0], g[0])
    assert same is g[0] and blocks.orthogonalise([]) == []
    flat = torch.zeros(1000)
    views = [flat[7:607].view(30, 20), flat[607:].view(-1)[:393][:300].view(15, 20)[:15]]
    assert blocks.orthogonalise(views[:1], [torch.zeros(30, 20, dtype=BF16)])[0].dtype == BF16


def test_orthogonalise_refuses(calls):
    g, other = torch.zeros(30, 20), torch.zeros(30, 20)
    bad = [
        lambda: blocks.orthogonalise(g[0]), lambda: blocks.orthogonalise(g.double()), lambda: blocks.orthogonalise([g, g[:20]]),
        lambda: blocks.orthogonalise([g, g.half()]), lambda: blocks.orthogonalise(g, accumulate=True), lambda: blocks.orthogonalise([g], g),
        lambda: blocks.orthogonalise([g, g], [g]), lambda: blocks.orthogonalise(g, g.t()), lambda: blocks.orthogonalise(g, steps=0),
        lambda: blocks.orthogonalise(g, coefficients=(1.0, 2.0)), lambda: blocks.orthogonalise(g.t()), lambda: blocks.orthogonalise(g[:0]),
        lambda: blocks.orthogonalise([g, g.clone()], [g.clone(), g.half()]), lambda: blocks.orthogonalise(g, g.to(torch.int32)),
        lambda: blocks.orthogonalise([g, g.clone()], [torch.zeros(30, 20)] * 2), lambda: blocks.orthogonalise(g, steps=2.5),
        lambda: blocks.orthogonalise([g, other], [other, g]), lambda: blocks.orthogonalise([g, other], [torch.zeros(30, 20), g]),
        lambda: blocks.orthogonalise([g, g], [g, other]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(dgs.DgsError) as err:
            call()
        assert err.value.code == EINVAL, i
    assert not calls
