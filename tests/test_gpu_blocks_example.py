"""examples/train_blocks.py: its gradients against autograd in fp32, and that a worker and its server train with them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_blocks", os.path.join(ROOT, "examples", "train_blocks.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def autograd(stack, x, dy):
    """The stack's flat gradient for loss = sum(y dy), in fp32 without checkpoints."""
    p = {k: v.clone().requires_grad_(True) for k, v in stack.p.items()}
    for b in range(stack.count):
        u = torch.nn.functional.layer_norm(x, (stack.width,), p[f"{b}.pre_weight"], p[f"{b}.pre_bias"])
        f = torch.nn.functional.gelu(u @ p[f"{b}.w1"].t() + p[f"{b}.b1"]) @ p[f"{b}.w2"].t()
        fh = f * torch.rsqrt(f.square().mean(1, keepdim=True) + 1e-5)
        x = x + p[f"{b}.gate"] * (fh * p[f"{b}.post_weight"] + p[f"{b}.post_bias"])
    (x * dy).sum().backward()
    return {k: v.grad for k, v in p.items()}, x


def test_gradients_near_autograd():
    """Codes are off by at most half a step, 1/128 of a run's largest value, bfloat16 values by 2^-9: each parameter's gradient
    points the same way within a few per cent."""
    m = example()
    stack = m.Stack(256, 512, 3, 640)
    x, dy = torch.randn(640, 256, device="cuda:0"), torch.randn(640, 256, device="cuda:0")
    want, y = autograd(stack, x, dy)
    got = stack.forward(x)
    stack.backward(dy)
    assert float((got - y).norm() / y.norm()) < 0.02
    for k, g in stack.g.items():
        w = want[k]
        cosine = float((g * w).sum() / (g.norm() * w.norm()))
        assert cosine > 0.99 and abs(float(g.norm() / w.norm()) - 1) < 0.05, (k, cosine, float(g.norm() / w.norm()))
    # a second pass adds the same again
    once = stack.grad.clone()
    stack.forward(x)
    stack.backward(dy)
    torch.testing.assert_close(stack.grad, 2 * once, rtol=1e-5, atol=1e-5 * float(once.abs().max()))


def test_training_lowers_the_loss():
    losses = example().train(steps=40, rows=1024, width=256, hidden=512, count=2, density=0.02, report=None)
    assert losses[-1] < 0.5 * losses[0], losses
