"""Further operators of `paper_1910_10929_amd.blocks` as cases that can be timed and compared.

What they are for: the two ends of a transformer worker's step that lie between its last block and the message that
`dgs.Context.worker_step` selects from a flat fp32 gradient:

  loss           the output layer with its loss: logits = x W^T + b, softmax cross entropy against one target a row.  Of a
                 large vocabulary the logits are by far the largest matrix of the step (8192 rows of 30522 in fp32: 1 GB), and
                 nobody needs them kept
  loss_grad      the same with its gradients: of x, for the last block, and of W and b, in fp32 for the flat buffer
  orthogonal     updates of weight matrices, orthogonalised by Newton-Schulz products before they are applied or sent: what a
                 matrix U S V^T keeps is U V^T, with singular values near 1

Loss: row t's loss is lse_t - logit_t[target_t] with lse_t = log sum exp logit_t; a row whose target is no entry of the
vocabulary (negative: padding) is left out, its loss is 0.  Gradients: for given dloss_t and dlse_t (what arrives at a row's loss and at
its lse; the second is how a penalty on lse comes in),

    dlogit_t = (dloss_t + dlse_t) softmax_t - dloss_t onehot(target_t),   dx = dlogit W,   dW = dlogit^T x,   db = sum_t dlogit_t

with dloss_t taken as 0 for a row that is left out.

Orthogonalised: X = G / (|G| + eps) with the Frobenius norm, then `STEPS` times, with A = X X^T, X = a X + (b A + c A^2) X
(X^T in place of X where there are more rows than columns).

Where `own` is false everything is computed in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------

def _loss(rows, cols, vocab, **more):
    c = {"op": "loss", "rows": rows, "cols": cols, "vocab": vocab, "type": "bf16", "bias": False, "left_out": 0.0, "penalty": 0.0,
         "pad": 0}
    c.update(more)
    return c


def _grad(rows, cols, vocab, **more):
    return _loss(rows, cols, vocab, **dict({"op": "loss_grad"}, **more))


def _ortho(count, rows, cols, **more):
    c = {"op": "orthogonal", "count": count, "rows": rows, "cols": cols, "type": "f32", "out": "f32"}
    c.update(more)
    return c


def listed():
    return [
        # one token's log probability, a transformer's width and vocabulary: latency, and the weights read once
        dict(_loss(1, 768, 30522), name="loss-token"),
        # a ragged batch of prompts that are scored, half precision, rows of a wider matrix, a part of them padding
        dict(_loss(1003, 1001, 5003, type="f16", bias=True, left_out=0.2, pad=3), name="loss-odd"),
        # an evaluation batch
        dict(_loss(16384, 768, 30522, left_out=0.1), name="loss-eval"),
        # a small model in fp32 throughout, odd sizes, with a penalty on lse
        dict(_grad(300, 333, 1009, type="f32", bias=True, left_out=0.1, penalty=1e-3), name="grad-small"),
        # a small half-precision step with a penalty on lse
        dict(_grad(2048, 1024, 32000, type="f16", penalty=1e-4), name="grad-half"),
        # an ordinary training step: a batch of 8192 tokens, a part of them padding
        dict(_grad(8192, 768, 30522, bias=True, left_out=0.1), name="grad-train"),
        # a wide model's training step
        dict(_grad(8192, 4096, 32768), name="grad-wide"),
        # one small matrix: latency
        dict(_ortho(1, 128, 128), name="ortho-small"),
        # a few odd-sized matrices
        dict(_ortho(5, 333, 1001), name="ortho-odd"),
        # the fused query/key/value projections of twelve blocks
        dict(_ortho(12, 2304, 768, out="bf16"), name="ortho-layers"),
        # four tall projections, for a flat fp32 update
        dict(_ortho(4, 4096, 1024), name="ortho-tall"),
        # a wide model's projection from a 16-bit update
        dict(_ortho(1, 4096, 4096, type="bf16", out="bf16"), name="ortho-wide"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rounded(rng, n, to):
    return (n + to - 1) // to * to if rng.random() < 0.6 else n


def draw(rng):
    """One more case: one row to 16,384 with 64 to 4096 columns and a vocabulary of 1000 to 131,072; one matrix to 24 of 64 to
    4096 rows and columns."""
    op = rng.choice(["loss", "loss_grad", "loss_grad", "orthogonal", "orthogonal"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "orthogonal":
        m, n = (_rounded(rng, _log_int(rng, 64, 4096), 32) for _ in range(2))
        # (fp32 results of the largest are three products each)
        most = 130_000_000_000 if kind != "f32" else 40_000_000_000
        count = max(1, min(_log_int(rng, 1, 24), most // (min(m, n) ** 2 * max(m, n))))
        return _ortho(count, m, n, type=rng.choice(["f32", "f32", kind]), out=kind)
    cols, vocab = _rounded(rng, _log_int(rng, 64, 4096), 32), _rounded(rng, _log_int(rng, 1000, 131072), 64)
    most = 1_000_000_000_000 if kind != "f32" else 150_000_000_000
    rows = max(1, min(_log_int(rng, 1, 16384), most // (cols * vocab)))
    return _loss(rows, cols, vocab, op=op, type=kind, bias=rng.random() < 0.4, left_out=rng.choice([0.0, 0.1, 0.4]),
                 penalty=rng.choice([0.0, 0.0, 1e-4]), pad=rng.choice([0, 0, 0, 64, 3]))


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------

def _prepare_loss(case, normal, uniform):
    rows, cols, vocab, dtype = case["rows"], case["cols"], case["vocab"], TYPES[case["type"]]
    s = {"case": case}
    s["weight"] = (normal(vocab, cols) * (1.5 / cols ** 0.5)).to(dtype)
    s["bias"] = 0.3 * normal(vocab) if case["bias"] else None
    # frequent entries first, and rows that point part of the way to their target's, as a trained model's do
    target = torch.floor(torch.exp(uniform(rows) * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)
    x = normal(rows, cols) + 2.0 * s["weight"].index_select(0, target).float()
    out = torch.zeros((rows, cols + case["pad"]), dtype=dtype, device=DEVICE)
    out[:, :cols] = x
    s["x"] = out[:, :cols]
    s["target"] = torch.where(uniform(rows) < case["left_out"], -100, target)
    if case["op"] == "loss_grad":
        # the mean over the rows that count; half precision with the loss scaled
        scale = (16384.0 if case["type"] == "f16" else 1.0) / max(1, rows - int(case["left_out"] * rows))
        s["dloss"] = torch.full((rows,), scale, dtype=torch.float32, device=DEVICE)
        s["penalty"] = 2.0 * case["penalty"] * scale
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, dtype=torch.float32, device=DEVICE, generator=gen)  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, dtype=torch.float32, device=DEVICE, generator=gen)  # noqa: E731
    if case["op"] != "orthogonal":
        return _prepare_loss(case, normal, uniform)
    count, rows, cols = case["count"], case["rows"], case["cols"]
    # gradients of linear layers, summed over twice as many rows as the smaller side has, channels of unlike scale: slices of
    # one flat buffer, a few values apart
    flat = torch.zeros(count * (rows * cols + 8), dtype=TYPES[case["type"]], device=DEVICE)
    given = []
    for i in range(count):
        deep = 2 * min(rows, cols)
        g = torch.matmul((normal(rows, deep) * torch.exp(0.5 * normal(rows, 1))), normal(deep, cols) * torch.exp(0.5 * normal(cols)))
        at = i * (rows * cols + 8)
        flat[at:at + rows * cols] = (g * (1e-3 / deep ** 0.5)).reshape(-1)
        given.append(flat[at:at + rows * cols].view(rows, cols))
    return {"case": case, "given": given}


# ----------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------

def _plain_loss(s):
    case = s["case"]
    x, w = s["x"].float(), s["weight"].float()
    logits = torch.matmul(x, w.t())
    if s["bias"] is not None:
        logits += s["bias"]
    top = logits.amax(1, keepdim=True)
    lse = torch.log(torch.exp(logits - top).sum(1)) + top.squeeze(1)
    counts = (s["target"] >= 0) & (s["target"] < case["vocab"])
    at = torch.where(counts, s["target"], 0).unsqueeze(1)
    out = {"loss": torch.where(counts, lse - logits.gather(1, at).squeeze(1), 0.0), "lse": lse}
    if case["op"] == "loss":
        return out
    dloss, dlse = torch.where(counts, s["dloss"], 0.0), s["penalty"] * lse
    d = torch.exp(logits - lse.unsqueeze(1)) * (dloss + dlse).unsqueeze(1)
    d.scatter_add_(1, at, -dloss.unsqueeze(1))
    out["dx"] = torch.matmul(d, w).to(s["x"].dtype)
    out["dweight"] = torch.matmul(d.t(), x)
    if s["bias"] is not None:
        out["dbias"] = d.sum(0)
    return out


def _plain_orthogonal(s):
    case = s["case"]
    a, b, c = COEFFICIENTS
    x = torch.stack(s["given"]).float()
    if case["rows"] > case["cols"]:
        x = x.transpose(1, 2).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        m = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * m + c * torch.matmul(m, m), x)
    if case["rows"] > case["cols"]:
        x = x.transpose(1, 2)
    return [v.contiguous() for v in x.to(TYPES[case["out"]])]


# ----------------------------------------------------------------------------
# the framework's operators
# ----------------------------------------------------------------------------

def _own_loss(s):
    from paper_1910_10929_amd import blocks
    case = s["case"]
    if "head" not in s:
        s["head"] = blocks.Head(s["weight"], s["bias"])         # the layer's handle, which a program keeps
    head = s["head"]
    loss, lse = head.forward(s["x"], s["target"])
    out = {"loss": loss, "lse": lse}
    if case["op"] == "loss":
        return out
    out["dweight"] = torch.empty((case["vocab"], case["cols"]), dtype=torch.float32, device=DEVICE)
    if s["bias"] is not None:
        out["dbias"] = torch.empty(case["vocab"], dtype=torch.float32, device=DEVICE)
    out["dx"] = head.backward(s["x"], s["target"], lse, dloss=s["dloss"], dlse=s["penalty"] * lse if s["penalty"] else None,
                              dweight=out["dweight"], dbias=out.get("dbias"))
    return out


def _own_orthogonal(s):
    from paper_1910_10929_amd import blocks
    case = s["case"]
    out = [torch.empty((case["rows"], case["cols"]), dtype=TYPES[case["out"]], device=DEVICE) for _ in s["given"]]
    return blocks.orthogonalise(s["given"], out, steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)


def run(state):
    if state["case"]["op"] == "orthogonal":
        return _own_orthogonal(state) if own else _plain_orthogonal(state)
    return _own_loss(state) if own else _plain_loss(state)


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------

def work(case):
    if case["op"] == "orthogonal":
        count, rows, cols = case["count"], case["rows"], case["cols"]
        m, n = min(rows, cols), max(rows, cols)
        # (of the symmetric products one half)
        return {"bytes": count * rows * cols * (BYTES[case["type"]] + BYTES[case["out"]]),
                "flops": count * STEPS * (m * m * n + m * m * m + 2 * m * m * n)}
    rows, cols, vocab, b = case["rows"], case["cols"], case["vocab"], BYTES[case["type"]]
    moved = (rows + vocab) * cols * b + rows * 16 + (4 * vocab if case["bias"] else 0)
    flops = 2 * rows * cols * vocab
    if case["op"] == "loss":
        return {"bytes": moved, "flops": flops}
    return {"bytes": moved + rows * cols * b + 4 * vocab * cols + rows * 4 + (4 * vocab if case["bias"] else 0), "flops": 3 * flops}


# ----------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    D = torch.float64
    if case["op"] == "orthogonal":
        a, b, c = COEFFICIENTS
        out = []
        for g in s["given"]:
            x = g.to(D)
            x = x / (torch.linalg.vector_norm(x) + EPS)
            tall = x.shape[0] > x.shape[1]
            eye = torch.eye(min(x.shape), dtype=D, device=DEVICE)
            for _ in range(STEPS):
                gram = x.t() @ x if tall else x @ x.t()
                p = torch.addmm(a * eye + b * gram, gram, gram, alpha=c)
                x = x @ p if tall else p @ x
            out.append(x)
        return out
    rows, cols, vocab = case["rows"], case["cols"], case["vocab"]
    x, w = s["x"].to(D), s["weight"].to(D)
    z = (w @ x.t()).t()
    if s["bias"] is not None:
        z = z + s["bias"].to(D)
    lse = torch.logsumexp(z, 1)
    live = torch.nonzero((s["target"] >= 0) & (s["target"] < vocab)).squeeze(1)
    loss = torch.zeros(rows, dtype=D, device=DEVICE)
    loss[live] = lse[live] - z[live, s["target"][live]]
    out = {"loss": loss, "lse": lse}
    if case["op"] == "loss":
        return out
    up = torch.zeros(rows, dtype=D, device=DEVICE)
    up[live] = s["dloss"].to(D)[live]
    z = torch.softmax(z, 1).mul_((up + s["penalty"] * lse).unsqueeze(1))
    z[live, s["target"][live]] -= up[live]
    out["dx"] = z @ w
    out["dweight"] = (x.t() @ z).t()
    if s["bias"] is not None:
        out["dbias"] = torch.ones(rows, dtype=D, device=DEVICE) @ z
    return out
