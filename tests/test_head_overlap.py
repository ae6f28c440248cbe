"""The output layer's two results in one buffer: refused before anything is enqueued (no GPU)."""
import pytest

from paper_1910_10929_amd import blocks, dgs

torch = pytest.importorskip("torch")

P = 1 << 20      # a pointer that is never followed


def forward(loss, lse):
    packed = blocks._HEAD.pack(4, 96, 100, 2, 8, 0, P, 96, P, 96, 0, P, loss, lse, 0, 0, 0, 0, 0, 0, 0, P, 1 << 40)
    return blocks.lib().dgs_head_forward(packed, None)


@pytest.mark.parametrize("loss, lse", [(P, P), (P + 12, P), (P, P + 4)])
def test_refused(loss, lse):
    assert forward(loss, lse) == dgs.DGS_EINVAL


def code_of(call):
    try:      # (an exception that a frame keeps would keep the frame's tensors until some later collection)
        call()
    except dgs.DgsError as e:
        return e.code
    return dgs.DGS_OK


@pytest.mark.gpu
def test_refused_by_the_binding():
    h = blocks.Head(torch.zeros(50, 40, device="cuda:0"))
    x, t, v = torch.zeros(6, 40, device="cuda:0"), torch.zeros(6, dtype=torch.int64, device="cuda:0"), torch.zeros(12, device="cuda:0")
    for loss, lse in ((v[:6], v[:6]), (v[:6], v[5:11])):
        assert code_of(lambda: h.forward(x, t, loss=loss, lse=lse)) == dgs.DGS_EINVAL
    loss, lse = h.forward(x, t, loss=v[:6], lse=v[6:])
    assert float((lse - torch.log(torch.tensor(50.0))).abs().max()) < 1e-5 and torch.equal(loss, lse)
