"""The end of a worker's step as it is used: the output layer's loss and gradients go into the flat fp32 gradient, its weight
matrices' gradients are orthogonalised into a flat update, and the worker step selects the message from that; against plain
computations in 64 bits, and captured into a graph.

Tolerances.  The gradients of one batch are off by what tests/test_gpu_head.py derives, here 2^-16 of their 2-norm at most (sums of 200 and 1000
terms, each off by a few 2^-20 of the magnitudes that went into it).  The orthogonalised update's own error is a few 2^-20 of its 2-norm for
matrices of this kind; a perturbation of a gradient, relative to its 2-norm, can grow by the iteration's slope at 0, 3.4445^5 = 485: 2^-16 + 485
2^-16 in all, taken against the update of the exact gradient; against that of the gradient as it is, 2^-16.  The selection is the oracle's,
on the bits that the worker step got."""
import numpy as np
import pytest

from paper_1910_10929_amd import blocks, dgs, synth

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV, D = "cuda:0", torch.float64


@pytest.fixture(scope="module", autouse=True)
def built():
    assert torch.cuda.is_available()
    dgs.lib()


class Model:
    """x -> x W1^T + b1 -> loss of the output layer W2, b2; parameters, gradients and updates in flat buffers."""

    def __init__(self, cols=96, vocab=1000, rows=200, seed=3):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        normal = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
        shapes = [(vocab, cols), (vocab,), (cols, cols)]
        self.offsets = synth.offsets_from_sizes(synth.sizes_of(shapes))
        n = int(self.offsets[-1])
        self.theta, self.grad, self.update = normal(n) * 0.1, torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        cut = lambda f: [f[int(a):int(e)].view(s) for s, a, e in zip(shapes, self.offsets, self.offsets[1:])]  # noqa: E731
        (self.w2, self.b2, self.w1), (self.g2, self.gb2, self.g1), (self.u2, self.ub2, self.u1) = cut(self.theta), cut(self.grad), cut(self.update)
        self.inputs = normal(rows, cols).bfloat16()
        self.targets = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
        self.targets[::9] = -100
        self.dloss = torch.full((rows,), 1.0 / float((self.targets >= 0).sum()), device=DEV)

    def gradients(self):
        x = torch.matmul(self.inputs, self.w1.bfloat16().t())
        head = blocks.Head(self.w2.bfloat16(), self.b2)
        loss, lse = head.forward(x, self.targets)
        dx = head.backward(x, self.targets, lse, dloss=self.dloss, dweight=self.g2, dbias=self.gb2, accumulate=True)
        blocks.weight_grad(dx, blocks.Checkpoint(*self.inputs.shape, device=DEV).encode(self.inputs), self.g1, accumulate=True)
        return x, loss, dx

    def orthogonal(self):
        blocks.orthogonalise(self.g2, self.u2, scale=0.2)
        blocks.orthogonalise(self.g1, self.u1, scale=0.2)
        self.ub2.copy_(self.gb2)


def exact64(g, scale):
    x = g / (g.norm() + 1e-7)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(5):
        m = x @ x.t()
        x = 3.4445 * x + (-4.7750 * m + 2.0315 * (m @ m)) @ x
    return scale * (x.t() if tall else x)


def test_step(oracle):
    m = Model()
    x, loss, dx = m.gradients()
    z = x.to(D) @ m.w2.bfloat16().to(D).t() + m.b2.to(D)
    counts = m.targets >= 0
    at = torch.where(counts, m.targets, 0)
    lse = torch.logsumexp(z, 1)
    want = torch.where(counts, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    assert float((loss.to(D) - want).abs().max()) < 2.0 ** -16 * float(lse.abs().max())
    up = torch.where(counts, m.dloss.to(D), 0.0)
    dz = torch.softmax(z, 1) * up[:, None]
    dz.scatter_add_(1, at[:, None], -up[:, None])
    for got, exact in ((m.g2, dz.t() @ x.to(D)), (m.gb2, dz.sum(0))):
        assert float((got.to(D) - exact).norm()) <= 2.0 ** -16 * float(exact.norm())
    assert float((dx.to(D) - dz @ m.w2.bfloat16().to(D)).norm()) <= 2.0 ** -8 * float(dx.to(D).norm())
    m.orthogonal()
    assert float((m.u2.to(D) - exact64(m.g2.to(D), 0.2)).norm()) <= 2.0 ** -16 * float(m.u2.to(D).norm())
    assert float((m.u1.to(D) - exact64(m.g1.to(D), 0.2)).norm()) <= 2.0 ** -16 * float(m.u1.to(D).norm())
    assert float((m.u2.to(D) - exact64(dz.t() @ x.to(D), 0.2)).norm()) <= 486 * 2.0 ** -16 * float(m.u2.to(D).norm())
    # the message is selected from the update
    n = int(m.offsets[-1])
    worker = dgs.Context(m.offsets, W=0, device=DEV)
    k = worker.nnz(0.01)
    state, idx, val = torch.zeros(n, device=DEV), torch.zeros(k, dtype=torch.int32, device=DEV), torch.zeros(k, device=DEV)
    s_ref = np.zeros(n, np.float32)
    for _ in range(3):
        worker.worker_step(m.update, state, 0.5, 0.7, 0.01, idx, val)
        wi, wv = oracle.worker_step(m.update.cpu().numpy(), s_ref, m.offsets, 0.5, np.float32(0.7), 0.01)
        assert np.array_equal(idx.cpu().numpy().view(np.uint32), wi) and np.array_equal(val.cpu().numpy(), wv)
        assert np.array_equal(state.cpu().numpy(), s_ref)
    worker.close()


def test_step_in_a_graph():
    """The same from a graph, replayed with other work between: the gradient is added to, the update written."""
    m = Model(seed=4)
    for _ in range(2):
        m.gradients()
        m.orthogonal()
    twice, update = m.grad.clone(), m.update.clone()
    m.grad.zero_()
    m.update.fill_(float("nan"))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        m.gradients()
        m.orthogonal()
    for _ in range(2):
        m.grad.zero_()
        graph.replay()
        float(torch.randn(1000, device=DEV).sum())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m.grad, twice) and torch.equal(m.update, update)


def test_learns_nothing_from_padding():
    """A batch of padding alone changes no gradient, and its updates are those of the gradient that is there."""
    m = Model(seed=5)
    m.gradients()
    before = m.grad.clone()
    m.targets.fill_(-1)
    _, loss, dx = m.gradients()
    assert torch.equal(m.grad, before) and bool((dx == 0).all()) and bool((loss == 0).all())
