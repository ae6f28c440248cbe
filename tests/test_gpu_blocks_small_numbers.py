"""Weight gradients of the smallest numbers of each type.

A value of dy goes through the matrix units in bfloat16 parts, whose smallest numbers are multiples of 2^-133: bfloat16 and half
are made of those, and so is an fp32 value from 2^-110 on; below, what is no multiple is left out, less than 2^-133 of each value.
Sums: as in test_gpu_blocks."""
import pytest

from paper_1910_10929_amd import blocks

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_blocks import BF16, D, DEV, EPS, F16, F32, Make, values64  # noqa: E402

# few rows; each of the tiles that these sizes take
SIZES = [(20, 16, 64), (64, 128, 128), (300, 130, 96), (1024, 256, 512)]


@pytest.mark.parametrize("rows, outs, cols", SIZES)
@pytest.mark.parametrize("dtype, unit, byte", [(BF16, -133, 248), (BF16, -126, 240), (F16, -24, 150), (F16, -16, 127), (F32, -133, 248), (F32, -120, 240)])
def test_whole_multiples_are_exact(rows, outs, cols, dtype, unit, byte):
    m = Make(rows + outs)
    dy = (torch.randint(-3, 4, (rows, outs), device=DEV, generator=m.g).to(D) * 2.0 ** unit).to(dtype)
    q = torch.randint(-15, 16, (rows, cols), device=DEV, generator=m.g, dtype=torch.int32).to(torch.int8)
    c = blocks.Checkpoint.of(q, torch.full((rows, (cols + 31) // 32), byte, dtype=torch.uint8, device=DEV))
    want = dy.to(D).t() @ values64(c)
    assert float(want.abs().max()) > 0
    dw, db = torch.empty(outs, cols, device=DEV), torch.empty(outs, device=DEV)
    blocks.weight_grad(dy, c, dw, db)
    assert torch.equal(dw.to(D), want) and torch.equal(db.to(D), dy.to(D).sum(0))


@pytest.mark.parametrize("rows, outs, cols", SIZES)
@pytest.mark.parametrize("power", [-100, -110, -112, -118, -126, -132, -140, -149])
def test_small_fp32_gradients(rows, outs, cols, power):
    m = Make(rows + outs)
    dy = ((torch.rand(rows, outs, dtype=D, device=DEV, generator=m.g) + 1) * 2.0 ** power).to(F32)
    dy *= torch.randint(0, 2, (rows, outs), device=DEV, generator=m.g).to(F32) * 2 - 1
    q = torch.randint(-127, 128, (rows, cols), device=DEV, generator=m.g, dtype=torch.int32).to(torch.int8)
    c = blocks.Checkpoint.of(q, torch.full((rows, (cols + 31) // 32), 248, dtype=torch.uint8, device=DEV))
    x, d = values64(c), dy.to(D)
    dw = torch.empty(outs, cols, device=DEV)
    blocks.weight_grad(dy, c, dw)
    size = (d.square().t() @ x.square()).sqrt()
    left_out = x.abs().sum(0) * 2.0 ** -133 if power < -110 else 0.0
    assert bool(((dw.to(D) - d.t() @ x).abs() <= (8 * rows ** 0.5 + 64) * EPS * size + left_out).all())
