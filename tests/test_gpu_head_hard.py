"""The output layer's gradients (blocks.Head) where numbers are hard, in norms, against the definition in 64 bits.

Tolerances.  A logit is a sum of `cols` products; fp32's additions round it to either side, by 2^-25 of partial sums of a size of 6 at most here,
so that it is off by some 2^-22 sqrt(cols), and by 2^-22 of its terms' 2-norm where operands are fp32; the exponential by 2^-22 of its argument of 30 at most, whose
multiple of log2 e is rounded to 2^-20.  That is what a value of dz = pull softmax - push onehot is off by relative to its terms, differently in every entry, and by 2^-22 since it is
held in two halves.  A gradient sums such errors as it sums the terms, and rounds its own additions, at most 8192 here, by 2^-24 sqrt(8192)
in all.  Together, relative to the gradient's 2-norm: 2^-22 sqrt(cols) + 2^-16.  (One half alone would leave 2^-12 / sqrt(3) = 2^-12.8, a part that is missing or
mistaken more; cols is at most 1024.)  Where entries are improbable, dz has steps of 2^-49 of its row's power of two: 2^-50 |x|^T power more for every entry."""
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


class Case:
    def __init__(self, rows, cols, vocab, dtype, lowered=0.0, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(1000 * seed + rows + 7 * cols + 11 * vocab)
        normal = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
        self.rows, self.cols, self.vocab, self.dtype = rows, cols, vocab, dtype
        self.x, self.w = normal(rows, cols).to(dtype), (normal(vocab, cols) / cols ** 0.5).to(dtype)
        self.bias = 0.3 * normal(vocab)
        self.bias[1::2] -= lowered
        self.targets = 2 * torch.randint(0, (vocab + 1) // 2, (rows,), device=DEV, generator=g)
        self.targets[torch.rand(rows, device=DEV, generator=g) < 0.2] = -100
        self.dloss, self.dlse = normal(rows), 0.1 * normal(rows)

    def run(self):
        head = blocks.Head(self.w, self.bias)
        lse = head.forward(self.x, self.targets)[1]
        dw, db = torch.full((self.vocab, self.cols), 7.0, device=DEV), torch.full((self.vocab,), 7.0, device=DEV)
        dx = head.backward(self.x, self.targets, lse, dloss=self.dloss, dlse=self.dlse, dweight=dw, dbias=db)
        return dx, dw, db

    def exact(self):
        x, w = self.x.to(D), self.w.to(D)
        z = (w @ x.t()).t() + self.bias.to(D)
        counts = self.targets >= 0
        up = torch.where(counts, self.dloss.to(D), 0.0)
        dz = torch.softmax(z, 1) * (up + self.dlse.to(D))[:, None]
        dz.scatter_add_(1, torch.where(counts, self.targets, 0)[:, None], -up[:, None])
        power = torch.exp2(torch.ceil(torch.log2(torch.maximum(up.abs(), (up + self.dlse.to(D)).abs()))))
        return dz @ w, dz.t() @ x, dz.sum(0), power

    def assert_near(self):
        dx, dw, db = self.run()
        want_dx, want_dw, want_db, power = self.exact()
        rel = 2.0 ** -22 * self.cols ** 0.5 + 2.0 ** -16
        if self.dtype == F32:
            assert float((dx.to(D) - want_dx).norm()) <= rel * float(want_dx.norm())
        else:      # (half a step of the result, and, of bfloat16, of the first halves alone)
            own = HALF[self.dtype] + (2.0 ** -11 if self.dtype == BF16 else 0.0)
            assert float((dx.to(D) - want_dx).norm()) <= (own + rel) * float(want_dx.norm()) + (2.0 ** -25 * dx.numel() ** 0.5 if self.dtype == F16 else 0.0)
        steps = 2.0 ** -50 * float((self.x.to(D).abs().t() @ power).norm())
        for part in (slice(0, None, 2), slice(1, None, 2)):
            n = len(range(self.vocab)[part]) ** 0.5
            off, size = float((dw[part].to(D) - want_dw[part]).norm()), float(want_dw[part].norm())
            assert off <= rel * size + n * steps, (off / size, rel, n * steps / size)
            off, size = float((db[part].to(D) - want_db[part]).norm()), float(want_db[part].norm())
            assert off <= rel * size, (off / size, rel)


# rows, columns, entries: every kind of tile among them
SIZES = [(40, 64, 200), (20, 96, 1000), (300, 333, 1009), (1000, 520, 4096), (512, 1024, 16384), (2048, 768, 8000), (8192, 256, 8000), (4096, 1024, 16384)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}")
def test_gradients_keep_22_bits(size, dtype):
    print(size, dtype, flush=True)
    Case(*size, dtype).assert_near()


@pytest.mark.parametrize("lowered", [10.0, 15.0, 20.0, 25.0])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("size", [(40, 64, 200), (20, 64, 200), (1000, 136, 3001)], ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}")
def test_improbable_entries(size, dtype, lowered):
    """Half of the entries lowered by their bias, to softmax of 2^-22 down to 2^-48: their weights' gradients keep their bits."""
    print(size, dtype, lowered, flush=True)
    Case(*size, dtype, lowered=lowered).assert_near()


@pytest.mark.parametrize("far", [1e9, 1e12, 1e25])
@pytest.mark.parametrize("size", [(32, 64, 300), (33, 64, 300), (1000, 96, 4000), (4096, 128, 16384)], ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}")
def test_one_weight_far_above_the_others(size, far):
    """fp32, in a column where x is 0, its entry taken out: every other logit is made of what is small beside it.  A logit of at most 60 here is
    off by 2^-25 60 sqrt(cols) and 2^-22 of its terms, less than 2^-14 with lse's own error; gradients as ever, but that W as it meets dx has steps of
    2^-50 of the largest, here on all entries of a row of dz, whose magnitudes sum to 2 of its power at most."""
    print(size, far, flush=True)
    c = Case(*size, F32)
    c.w.mul_(4.0)
    c.x[:, 5] = 0.0
    c.w[7, 5], c.bias[7] = far, -float("inf")
    want = torch.logsumexp((c.w.to(D) @ c.x.to(D).t()).t() + c.bias.to(D), 1)
    lse = blocks.Head(c.w, c.bias).forward(c.x, c.targets)[1]
    assert float((lse.to(D) - want).abs().max()) <= 2.0 ** -14
    dx, dw, db = c.run()
    want_dx, want_dw, want_db, power = c.exact()
    rel = 2.0 ** -20 * c.cols ** 0.5 + 2.0 ** -16
    assert float((dw.to(D) - want_dw).norm()) <= rel * float(want_dw.norm())
    assert float((db.to(D) - want_db).norm()) <= rel * float(want_db.norm())
    assert float((dx.to(D) - want_dx).norm()) <= rel * float(want_dx.norm()) + 2.0 ** -50 * far * 2.0 * float(power.norm()) * c.cols ** 0.5
