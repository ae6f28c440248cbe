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
