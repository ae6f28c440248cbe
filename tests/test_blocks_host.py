"""Host side of the training blocks' C ABI, without a GPU: every symbol of the header is exported and bound, workspace sizes,
and what the calls refuse -- all of it before anything is enqueued."""
import ctypes
import os
import re

import pytest

from paper_1910_10929_amd import blocks, dgs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ENOMEM, ENOTSUP = dgs.DGS_EINVAL, dgs.DGS_ENOMEM, dgs.DGS_ENOTSUP
P = 1 << 20      # a pointer that is never followed


def _declared_symbols():
    text = open(os.path.join(ROOT, "include", "dgs_blocks.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(dgs_[a-z_]+)\s*\(", text)))


def test_header_symbols_are_exported():
    names = _declared_symbols()
    L = blocks.lib()
    assert names == sorted(blocks.EXPORTS)
    for name in names:
        assert hasattr(L, name), f"libdgs.so does not export {name}"


def test_workspace_sizes():
    L = blocks.lib()
    assert L.dgs_edge_backward_workspace(0, 768, 0) == 0
    assert L.dgs_edge_backward_workspace(5, 0, 0) == 0
    assert L.dgs_edge_backward_workspace(5, 16385, 0) == 0
    # at least one row of any type for each of the five sums
    for rows, cols, per in ((1, 1, 0), (1, 768, 1), (8192, 768, 512), (100000, 64, 1), (3, 16384, 2), (70000, 512, 37)):
        assert L.dgs_edge_backward_workspace(rows, cols, per) >= 20 * cols
    assert L.dgs_checkpoint_weight_grad_workspace(100, 0, 5, 0) == 0
    assert L.dgs_checkpoint_weight_grad_workspace(100, 5, 0, 0) == 0
    assert L.dgs_checkpoint_weight_grad_workspace(100, 5, 5, 3) == 0
    assert L.dgs_checkpoint_weight_grad_workspace(0, 5, 7, 2) >= 4 * 5 * 7
    # partial sums stay in proportion to the result: of the order of the chip's accumulators at most, or a few copies
    for rows, outs, cols in ((32768, 4096, 4096), (65536, 64, 64), (1, 8192, 8192), (8192, 2304, 768)):
        assert L.dgs_checkpoint_weight_grad_workspace(rows, outs, cols, 2) <= max(160 << 20, 6 * 4 * outs * cols)


# -- dgs_edge_forward -------------------------------------------------------------

EDGE = dict(cols=768, post=1, pre=2, post_eps=1e-5, pre_eps=1e-5, skip=1.0, branch=1.0, pw=P, pb=P, nw=P, nb=P)
FWD = dict(rows=4, per=0, stream=2, type=2, gate_type=0, x=P, xs=768, f=P, fs=768, gate=0, gs=0, xo=P, xos=768, u=P, us=768,
           pc=0, pcs=0, pe=0, pes=0, nc=0, ncs=0, ne=0, nes=0, stats=0)


def _edge(**k):
    e = dict(EDGE, **{n: v for n, v in k.items() if n in EDGE})
    return blocks._EDGE.pack(*e.values())


def forward(**k):
    a = dict(FWD, **{n: v for n, v in k.items() if n in FWD})
    assert set(k) <= set(FWD) | set(EDGE)
    v = list(a.values())
    return blocks.lib().dgs_edge_forward(_edge(**k), blocks._FORWARD.pack(*v[:5], 0, *v[5:]), None)


@pytest.mark.parametrize("code, change", [
    (EINVAL, dict(cols=0)),
    (EINVAL, dict(post=3)), (EINVAL, dict(pre=-1)),
    (EINVAL, dict(post_eps=0.0)), (EINVAL, dict(pre_eps=-1.0)), (EINVAL, dict(pre_eps=float("nan"))), (EINVAL, dict(post_eps=float("inf"))),
    (EINVAL, dict(skip=float("nan"))), (EINVAL, dict(branch=float("nan"))),
    (EINVAL, dict(pw=P + 2)), (EINVAL, dict(nb=P + 1)),
    (EINVAL, dict(stream=3)), (EINVAL, dict(type=-1)),
    (EINVAL, dict(x=0)), (EINVAL, dict(x=P + 1)), (EINVAL, dict(xs=767)), (EINVAL, dict(xs=1 << 32)),
    (EINVAL, dict(fs=767)), (EINVAL, dict(xo=0)), (EINVAL, dict(xos=1)),
    (EINVAL, dict(u=0)), (EINVAL, dict(us=700)),
    (EINVAL, dict(pre=0)),                                  # u without a norm
    (EINVAL, dict(pre=0, u=0, nc=P, ncs=768, ne=P, nes=24)),     # a checkpoint of a norm that is not there
    (EINVAL, dict(f=0)),                                    # x_out without a branch
    (EINVAL, dict(f=0, xo=0)),                              # a norm of a branch that is not there
    (EINVAL, dict(f=0, xo=0, post=0, pw=0, pb=0, gate=P, gs=768, per=1)),
    (EINVAL, dict(f=0, xo=0, post=0, pre=0, u=0)),          # nothing to do
    (EINVAL, dict(gate=P, gs=768, per=0, gate_type=2)),
    (EINVAL, dict(gate=P, gs=768, per=1, gate_type=1)),     # neither fp32 nor the branch's type
    (EINVAL, dict(gate=P, gs=767, per=1, gate_type=2)),
    (EINVAL, dict(gate=P + 2, gs=768, per=1, gate_type=0)),
    (EINVAL, dict(pc=P, pcs=768, pe=0, pes=24)), (EINVAL, dict(pc=P, pcs=767, pe=P, pes=24)), (EINVAL, dict(nc=P, ncs=768, ne=P, nes=23)),
    (EINVAL, dict(stats=P + 1)),
    (ENOTSUP, dict(cols=16385, xs=16385, fs=16385, xos=16385, us=16385)),
    (ENOTSUP, dict(stream=2, type=1)), (ENOTSUP, dict(stream=1, type=2)), (ENOTSUP, dict(stream=2, type=0)),
    (ENOTSUP, dict(rows=1 << 31)),
])
def test_forward_refuses(code, change):
    assert forward(**change) == code


def test_no_rows_is_no_work():
    assert forward(rows=0) == 0
    L = blocks.lib()
    codes = blocks._CODES.pack(P, 100, P, 4)
    assert L.dgs_checkpoint_encode(0, 100, 0, None, 0, codes, None) == 0
    assert L.dgs_checkpoint_decode(0, 100, codes, None, None, 0, None, 0, None) == 0


def test_null_structures():
    L = blocks.lib()
    assert L.dgs_edge_forward(None, None, None) == EINVAL
    assert L.dgs_edge_backward(None, None, None) == EINVAL
    assert L.dgs_checkpoint_weight_grad(None, None) == EINVAL
    assert L.dgs_checkpoint_encode(1, 1, 0, P, 1, None, None) == EINVAL
    assert L.dgs_checkpoint_decode(1, 1, None, None, None, 0, P, 1, None) == EINVAL


# -- dgs_edge_backward ------------------------------------------------------------

BWD = dict(rows=4, per=0, stream=2, type=2, gate_type=0, accumulate=0, d=P, ds=768, du=P, dus=768, gate=0, gs=0, f=0, fs=0, x=0, xs=0,
           pc=P, pcs=768, pe=P, pes=24, nc=P, ncs=768, ne=P, nes=24, stats=P, dx=P, dxs=768, df=P, dfs=768, dg=0, dgs=0,
           gpw=P, gpb=P, gnw=P, gnb=P, ws=P, wsb=1 << 30)


def backward(**k):
    a = dict(BWD, **{n: v for n, v in k.items() if n in BWD})
    assert set(k) <= set(BWD) | set(EDGE)
    return blocks.lib().dgs_edge_backward(_edge(**k), blocks._BACKWARD.pack(*a.values()), None)


VALUES = dict(pc=0, pcs=0, pe=0, pes=0, nc=0, ncs=0, ne=0, nes=0, f=P, fs=768, x=P, xs=768)


@pytest.mark.parametrize("code, change", [
    (EINVAL, dict(cols=0)), (EINVAL, dict(stream=7)),
    (EINVAL, dict(pre=0, nw=0, nb=0)),                      # du without a norm
    (EINVAL, dict(pc=0, pe=0)),                             # a norm of a branch that is not there
    (EINVAL, dict(post=0, pc=0, pe=0)),                     # df without a branch
    (EINVAL, dict(dg=P, dgs=768)),                          # dgate without a gate
    (EINVAL, dict(gate=P, gs=768, per=0)), (EINVAL, dict(gate=P, gs=768, per=2, dg=P, dgs=700)),
    (EINVAL, dict(ds=700)), (EINVAL, dict(dus=1)), (EINVAL, dict(dxs=2)), (EINVAL, dict(dfs=767)), (EINVAL, dict(dx=P + 1)),
    (EINVAL, dict(f=P, fs=768)),                            # both kinds of one norm
    (EINVAL, dict(nc=0, ne=0, x=P, xs=768)),                # one norm in codes, the other in values
    (EINVAL, dict(VALUES, fs=700)), (EINVAL, dict(VALUES, x=0)),
    (EINVAL, dict(pes=23)), (EINVAL, dict(ne=0)),
    (EINVAL, dict(stats=0)), (EINVAL, dict(stats=P + 2)),
    (EINVAL, dict(gpw=P + 1)), (EINVAL, dict(gnb=P + 2)),
    (EINVAL, dict(ws=0)), (EINVAL, dict(ws=P + 8)), (ENOMEM, dict(wsb=100)),
    (ENOTSUP, dict(stream=1)), (ENOTSUP, dict(rows=1 << 31)),
    (ENOTSUP, dict(cols=16400, ds=16400, dus=16400, dxs=16400, dfs=16400, pcs=16400, ncs=16400, pes=600, nes=600)),
])
def test_backward_refuses(code, change):
    assert backward(**change) == code


# -- checkpoints and the weight gradient ----------------------------------------------

@pytest.mark.parametrize("change", [dict(cols=0), dict(type=3), dict(x=0), dict(x=P + 1), dict(stride=99), dict(codes=0), dict(exps=0),
                                    dict(cs=99), dict(es=3)])
def test_encode_and_decode_refuse(change):
    a = dict(dict(cols=100, type=2, x=P, stride=100, codes=P, exps=P, cs=100, es=4), **change)
    codes = blocks._CODES.pack(a["codes"], a["cs"], a["exps"], a["es"])
    L = blocks.lib()
    assert L.dgs_checkpoint_encode(3, a["cols"], a["type"], a["x"], a["stride"], codes, None) == EINVAL
    assert L.dgs_checkpoint_decode(3, a["cols"], codes, None, None, a["type"], a["x"], a["stride"], None) == EINVAL


def test_decode_refuses_vectors_and_sizes():
    codes = blocks._CODES.pack(P, 100, P, 4)
    L = blocks.lib()
    assert L.dgs_checkpoint_decode(3, 100, codes, P + 1, None, 0, P, 100, None) == EINVAL
    assert L.dgs_checkpoint_decode(3, 100, codes, None, P + 2, 0, P, 100, None) == EINVAL
    big = blocks._CODES.pack(P, 1 << 20, P, 1 << 20)
    assert L.dgs_checkpoint_encode(0xFFFFFFFF, 1 << 20, 0, P, 1 << 20, big, None) == ENOTSUP


GRAD = dict(rows=64, outs=96, cols=100, type=2, accumulate=0, dy=P, dys=96, codes=P, cs=100, exps=P, es=4, scale=0, shift=0, dw=P, dws=100,
            db=0, ws=P, wsb=1 << 30)


@pytest.mark.parametrize("code, change", [
    (EINVAL, dict(outs=0)), (EINVAL, dict(cols=0)), (EINVAL, dict(type=4)),
    (EINVAL, dict(dy=0)), (EINVAL, dict(dy=P + 1)), (EINVAL, dict(dys=95)), (EINVAL, dict(cs=99)), (EINVAL, dict(es=3)), (EINVAL, dict(codes=0)),
    (EINVAL, dict(dw=0)), (EINVAL, dict(dw=P + 2)), (EINVAL, dict(dws=99)), (EINVAL, dict(scale=P + 1)), (EINVAL, dict(shift=P + 2)),
    (EINVAL, dict(db=P + 1)), (EINVAL, dict(ws=0)), (EINVAL, dict(ws=P + 4)), (ENOMEM, dict(wsb=64)),
    (ENOTSUP, dict(dys=1 << 28)), (ENOTSUP, dict(cs=1 << 28)), (ENOTSUP, dict(rows=1 << 31)),
])
def test_weight_grad_refuses(code, change):
    v = list(dict(GRAD, **change).values())
    assert blocks.lib().dgs_checkpoint_weight_grad(blocks._GRAD.pack(*v[:5], 0, *v[5:]), None) == code


# -- the binding ----------------------------------------------------------------------

def test_binding_refuses_host_tensors_and_bad_layers():
    import torch
    x = torch.zeros(4, 32)
    for call in (lambda: blocks.Edge(32, pre="batch"), lambda: blocks.Edge(32, post_weight=x[0]), lambda: blocks.Edge(32, pre_bias=x[0]),
                 lambda: blocks.Edge(32, pre="rms", pre_weight=x[0]), lambda: blocks.Edge(32, pre="rms").forward(x),
                 lambda: blocks.Checkpoint(4, 32, device="cpu"), lambda: blocks.weight_grad(x, None, x)):
        with pytest.raises(dgs.DgsError) as e:
            call()
        assert e.value.code == EINVAL
