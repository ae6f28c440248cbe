"""A worker and its server train a stack of residual blocks on one GPU:

    python examples/train_blocks.py [--steps 60] [--rows 4096] [--width 768] [--blocks 4] [--density 0.01]

Every block is u = N_pre(x), h = u W1^T, a = gelu(h), f = a W2^T, x = x + gate * N_post(f), with the residual stream in fp32
and the branch in bfloat16.  What lies between two blocks is one call of `blocks.Edge`, forward and backward.  For the backward
pass a block keeps 8-bit checkpoints alone -- of the normalised stream, of h, of a and of the normalised branch -- and both weight
gradients are read from them (`blocks.weight_grad`), straight into the flat fp32 gradient that `dgs.Context.worker_step` sends
the largest entries of.  The server answers with the largest entries of what the worker has not seen yet.

The task is synthetic: the outputs of a random stack of the same kind.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1910_10929_amd import blocks, dgs, synth  # noqa: E402


class Stack:
    """The blocks on a flat fp32 parameter buffer, with their gradients in another of the same layout."""

    def __init__(self, width, hidden, count, rows, device="cuda:0", seed=0):
        self.width, self.hidden, self.count, self.rows, self.device = width, hidden, count, rows, device
        names, shapes = [], []
        for b in range(count):
            names += [f"{b}.{n}" for n in ("pre_weight", "pre_bias", "w1", "b1", "w2", "post_weight", "post_bias", "gate")]
            shapes += [(width,), (width,), (hidden, width), (hidden,), (width, hidden), (width,), (width,), (1, width)]
        self.offsets = synth.offsets_from_sizes(synth.sizes_of(shapes))
        n = int(self.offsets[-1])
        self.theta = torch.zeros(n, device=device)
        self.grad = torch.zeros(n, device=device)
        cut = lambda flat: {k: flat[int(a):int(e)].view(s) for k, s, a, e in zip(names, shapes, self.offsets, self.offsets[1:])}  # noqa: E731
        self.p, self.g = cut(self.theta), cut(self.grad)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        for k, v in self.p.items():
            if k.endswith("_weight"):
                v.fill_(1.0)
            elif k.endswith("gate"):
                v.fill_(0.5)
            elif v.dim() == 2:
                v.copy_(torch.randn(v.shape, device=device, generator=gen) / v.shape[1] ** 0.5)
        p = lambda b, n: self.p.get(f"{b}.{n}")  # noqa: E731
        # edge b lies before block b: behind block b - 1, if there is one, and before block b, if there is one
        self.edges = [blocks.Edge(width, post="rms" if b > 0 else None, pre="layer" if b < count else None,
                                  post_weight=p(b - 1, "post_weight"), post_bias=p(b - 1, "post_bias"),
                                  pre_weight=p(b, "pre_weight"), pre_bias=p(b, "pre_bias")) for b in range(count + 1)]
        # (no branch ends at the first edge, no block begins behind the last one)
        self.saved = [blocks.Saved(rows, width, device=device, post=blocks.Checkpoint(rows, width, device) if b > 0 else None,
                                   pre=blocks.Checkpoint(rows, width, device) if b < count else None) for b in range(count + 1)]
        self.kept = [(blocks.Checkpoint(rows, hidden, device), blocks.Checkpoint(rows, hidden, device)) for _ in range(count)]

    def kept_bytes(self):
        """What the forward pass leaves for the backward pass."""
        c = [k for pair in self.kept for k in pair] + [k for s in self.saved for k in (s.post, s.pre) if k is not None]
        return sum(k.codes.numel() + k.exps.numel() for k in c) + sum(s.stats.numel() * 4 for s in self.saved)

    def forward(self, x):
        f = None
        for b in range(self.count):
            gate = self.p[f"{b - 1}.gate"] if b else None
            x, u = self.edges[b].forward(x, f, gate=gate, u=torch.empty_like(x, dtype=torch.bfloat16) if f is None else None,
                                         save=self.saved[b])
            h = torch.addmm(self.p[f"{b}.b1"].bfloat16(), u, self.p[f"{b}.w1"].bfloat16().t())
            a = torch.nn.functional.gelu(h)
            self.kept[b][0].encode(h)
            self.kept[b][1].encode(a)
            f = torch.matmul(a, self.p[f"{b}.w2"].bfloat16().t())
        return self.edges[-1].forward(x, f, gate=self.p[f"{self.count - 1}.gate"], save=self.saved[-1])[0]

    def backward(self, dx):
        """Adds to `grad`; dx: the gradient of the stack's output."""
        du = None
        for b in range(self.count, -1, -1):
            g = lambda n, at: self.g.get(f"{at}.{n}")  # noqa: E731
            more = {}
            if b > 0:
                more = dict(gate=self.p[f"{b - 1}.gate"], dgate=g("gate", b - 1), post_weight_grad=g("post_weight", b - 1),
                            post_bias_grad=g("post_bias", b - 1))
            if b < self.count:
                more.update(pre_weight_grad=g("pre_weight", b), pre_bias_grad=g("pre_bias", b))
            else:
                more["du"] = None
            dx, df = self.edges[b].backward(self.saved[b], dx_out=dx, du=more.pop("du", du), accumulate=True, **more)
            if b == 0:
                return dx
            h, a = self.kept[b - 1]
            blocks.weight_grad(df, a, g("w2", b - 1), accumulate=True)
            da = torch.matmul(df, self.p[f"{b - 1}.w2"].bfloat16())
            dh = torch.ops.aten.gelu_backward(da, h.decode(dtype=torch.bfloat16))
            # the block's input was the normalised stream times the norm's weight plus its bias
            blocks.weight_grad(dh, self.saved[b - 1].pre, g("w1", b - 1), g("b1", b - 1), scale=self.p[f"{b - 1}.pre_weight"],
                               shift=self.p[f"{b - 1}.pre_bias"], accumulate=True)
            du = torch.matmul(dh, self.p[f"{b - 1}.w1"].bfloat16())


def train(steps=60, rows=4096, width=768, hidden=2304, count=4, density=0.01, lr=0.002, momentum=0.7, micro=2, report=print):
    """Losses step by step.  The gradient of a step is added up over `micro` batches."""
    torch.manual_seed(0)
    dev = "cuda:0"
    teacher, model = Stack(width, hidden, count, rows, dev, seed=1), Stack(width, hidden, count, rows, dev, seed=2)
    n = int(model.offsets[-1])
    worker, server = dgs.Context(model.offsets, W=0, device=dev), dgs.Context(model.offsets, W=1, device=dev)
    k = worker.nnz(density)
    velocity, diff = torch.zeros(n, device=dev), torch.zeros(1, n, device=dev)
    server.server_attach(diff)
    pairs = lambda: (torch.zeros(k, dtype=torch.int32, device=dev), torch.zeros(k, device=dev))  # noqa: E731
    (idx, val), (reply_idx, reply_val) = pairs(), pairs()
    losses = []
    for step in range(steps):
        model.grad.zero_()
        loss = 0.0
        for _ in range(micro):
            x = torch.randn(rows, width, device=dev)
            want = teacher.forward(x.clone())
            error = model.forward(x) - want
            loss = loss + error.square().mean() / micro
            model.backward(error * (2.0 / (rows * micro)))
        worker.worker_step(model.grad, velocity, lr, momentum, density, idx, val)
        server.server_push(None, 0, idx, val, k)
        server.server_pull(0, density, reply_idx, reply_val)
        worker.apply_sparse(model.theta, reply_idx, reply_val, k)
        losses.append(loss)
        if report and (step % 10 == 0 or step == steps - 1):
            report(f"step {step:3d}  loss {float(loss):.5f}")
    losses = [float(v) for v in losses]
    worker.close()
    server.close()
    if report:
        full = rows * (2 * width * (count + 1) + 2 * hidden * count) * 2
        report(f"{n / 1e6:.1f} M parameters, {k} sent a step; {model.kept_bytes() / 1e6:.1f} MB kept for the backward pass, {full / 1e6:.1f} MB in 16 bits")
    return losses


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--steps", type=int, default=60)
    a.add_argument("--rows", type=int, default=4096)
    a.add_argument("--width", type=int, default=768)
    a.add_argument("--hidden", type=int, default=2304)
    a.add_argument("--blocks", type=int, default=4)
    a.add_argument("--density", type=float, default=0.01)
    a = a.parse_args()
    train(a.steps, a.rows, a.width, a.hidden, a.blocks, a.density)


if __name__ == "__main__":
    main()
