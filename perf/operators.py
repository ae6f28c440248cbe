"""The operators of `paper_1910_10929_amd.blocks` as cases that can be timed and compared.

What they are for: a worker that trains a transformer and sends its gradient through
`dgs.Context.worker_step` keeps its parameters and its gradient in flat fp32 buffers.  The
operators here are the memory-bound part of its blocks, and the part that decides how much the
forward pass has to keep for the backward pass:

  edge           what lies between two blocks: the branch's output is normalised, gated, scaled and
                 added to the residual stream, and the stream is normalised for the next branch;
                 in training both normalised values are kept as 8-bit checkpoints
  edge_backward  its gradients, from the checkpoints (or from values kept in full)
  checkpoint     a tensor into 8 bits and back
  weight_grad    a linear layer's weight and bias gradient, its input read from the checkpoint

Checkpoint of a matrix: every run of 32 columns of a row shares a power of two 2^e, the smallest
for which all of the run rounds into [-127, 127] (e from -126 to 121); codes are whole numbers.
A run that holds an infinity or NaN reads as NaN.  What a checkpoint stands for, q 2^e, is exact in
bfloat16, and that is how it is returned here.

Where `own` is false everything is computed in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
RUN = 32
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------

def _edge(rows, cols, **more):
    c = {"op": "edge", "rows": rows, "cols": cols, "type": "bf16", "stream": "bf16", "post": "rms", "pre": "rms",
         "bias": False, "rows_per_gate": 0, "gate_type": "bf16", "save": "none", "pad": 0, "skip": 1.0, "branch": 1.0}
    c.update(more)
    return c


def _back(rows, cols, **more):
    return _edge(rows, cols, **dict({"op": "edge_backward", "save": "checkpoint"}, **more))


def _checkpoint(rows, cols, **more):
    c = {"op": "checkpoint", "rows": rows, "cols": cols, "type": "bf16", "affine": False, "pad": 0}
    c.update(more)
    return c


def _grad(rows, outs, cols, **more):
    c = {"op": "weight_grad", "rows": rows, "outs": outs, "cols": cols, "type": "bf16", "affine": "scale", "bias": True,
         "pad": 0}
    c.update(more)
    return c


def listed():
    return [
        # one token of a served model: a single launch, latency
        dict(_edge(1, 768, post="layer", pre="layer", bias=True), name="edge-token"),
        # a batch of odd-sized prompts, modulated per sequence of 59 tokens, half precision, rows of a wider matrix
        dict(_edge(1003, 1001, type="f16", stream="f16", rows_per_gate=59, gate_type="f16", pad=3, branch=0.5),
             name="edge-prompts-odd"),
        # an ordinary training step on the transformer's width: fp32 residual stream, learned gate per channel
        dict(_edge(8192, 768, post="layer", pre="layer", bias=True, stream="f32", rows_per_gate=8192, gate_type="f32",
                   save="checkpoint"), name="edge-train"),
        # a wide model's training step, gates per token
        dict(_edge(16384, 4096, rows_per_gate=1, save="checkpoint"), name="edge-train-wide"),
        # the backward of the ordinary step, gate per sequence of 512 tokens
        dict(_back(8192, 768, post="layer", pre="layer", bias=True, stream="f32", rows_per_gate=512), name="back-train"),
        # a small odd-sized layer in fp32 whose values were kept in full
        dict(_back(777, 1001, type="f32", stream="f32", post="layer", pre="rms", bias=True, rows_per_gate=37,
                   gate_type="f32", save="values"), name="back-odd"),
        # the backward of the wide step, learned gate per channel
        dict(_back(16384, 4096, rows_per_gate=16384, gate_type="f32", branch=0.7), name="back-wide"),
        # a small fp32 activation
        dict(_checkpoint(64, 1000, type="f32"), name="checkpoint-small"),
        # the activations of a whole step: 150 M values
        dict(_checkpoint(65536, 2304), name="checkpoint-large"),
        # the fused query/key/value projection behind a layer norm
        dict(_grad(8192, 2304, 768, affine="both"), name="grad-qkv"),
        # a small odd-sized projection with fp32 gradients
        dict(_grad(1500, 1001, 333, type="f32", affine="none"), name="grad-odd"),
        # a wide model's projection
        dict(_grad(32768, 4096, 4096, bias=False), name="grad-wide"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any of the operators, one row to 65,536, 64 to 8192 columns."""
    op = rng.choice(["edge", "edge", "edge_backward", "edge_backward", "checkpoint", "weight_grad", "weight_grad"])
    cols = _log_int(rng, 64, 8192)
    if rng.random() < 0.6:
        cols = (cols + 31) // 32 * 32
    rows = _log_int(rng, 1, 65536)
    pad = rng.choice([0, 0, 0, 64, 3])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "weight_grad":
        outs = _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            outs = (outs + 63) // 64 * 64
        rows = max(1, min(rows, 500_000_000_000 // (outs * cols)))
        if kind == "f32":
            rows = max(1, rows // 3)
        return _grad(rows, outs, cols, type=kind, affine=rng.choice(["none", "scale", "both"]), bias=rng.random() < 0.6, pad=pad)
    rows = max(1, min(rows, 60_000_000 // cols))
    if op == "checkpoint":
        return _checkpoint(rows, cols, type=kind, affine=rng.random() < 0.3, pad=pad)
    gate = rng.choice(["none", "token", "sequence", "sequence", "channel"])
    rpg = {"none": 0, "token": 1, "sequence": _log_int(rng, 2, 2048), "channel": rows}[gate]
    more = dict(type=kind, stream=rng.choice([kind, "f32"]), post=rng.choice(["rms", "layer", "none"]),
                pre=rng.choice(["rms", "layer"]), bias=rng.random() < 0.5, rows_per_gate=rpg,
                gate_type="f32" if gate == "channel" else kind, pad=pad,
                skip=rng.choice([1.0, 1.0, 1.5]), branch=rng.choice([1.0, 0.7]))
    if op == "edge":
        return _edge(rows, cols, save=rng.choice(["none", "checkpoint"]), **more)
    return _back(rows, cols, save=rng.choice(["checkpoint", "checkpoint", "values"]), **more)


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------

class _Make:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.gen = torch.Generator(device=DEVICE)
        self.gen.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, dtype=torch.float32, device=DEVICE, generator=self.gen)

    def activation(self, rows, cols, dtype, pad=0, scale=1.0):
        """Normal values whose channels differ in scale, one in 64 of them six times the others'; the first
        columns of rows that are `pad` values longer."""
        width = torch.exp(0.3 * self.normal(cols))
        width *= torch.where(torch.rand(cols, device=DEVICE, generator=self.gen) < 1.0 / 64.0, 6.0, 1.0)
        out = torch.zeros((rows, cols + pad), dtype=dtype, device=DEVICE)
        out[:, :cols] = self.normal(rows, cols).mul_(width * scale)
        return out[:, :cols]

    def weight(self, cols):
        return 1.0 + 0.2 * self.normal(cols)

    def bias(self, cols):
        return 0.1 * self.normal(cols)

    def gate(self, rows, cols, dtype):
        return (0.5 + 0.5 * self.normal(rows, cols)).to(dtype)


def _codes(v):
    """The checkpoint of fp32 values: (codes int8, exponent bytes uint8).  From the bits of a run's largest magnitude:
    its exponent less 6, one more where the mantissa is at least 127.5 / 64 (what would round to 128)."""
    rows, cols = v.shape
    runs = (cols + RUN - 1) // RUN
    p = torch.nn.functional.pad(v, (0, runs * RUN - cols)).view(rows, runs, RUN)
    top = (p.view(torch.int32) & 0x7FFFFFFF).amax(2)
    byte = (((top + 0x10000) >> 23) - 6).clamp(1, 248)
    scale = ((254 - byte) << 23).view(torch.float32)            # 2^-e, e = byte - 127
    q = torch.round(p * scale.unsqueeze(2)).clamp(-127.0, 127.0)
    bad = top >= 0x7F800000
    byte = torch.where(bad, 255, byte)
    q = torch.where(bad.unsqueeze(2), 0.0, q)
    return q.view(rows, -1)[:, :cols].to(torch.int8).contiguous(), byte.to(torch.uint8)


def _values(q, e):
    """What a checkpoint stands for, in fp32."""
    byte = e.to(torch.int32).repeat_interleave(RUN, 1)[:, :q.shape[1]]
    scale = torch.where(byte == 255, float("nan"), (byte << 23).view(torch.float32))
    return q.to(torch.float32) * scale


def _norm(v, kind, eps):
    """Normalised values, mean and 1 / deviation of each row."""
    if kind == "none":
        return v, None, None
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    d = v - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + eps)
    return d * rstd, mean, rstd


EPS = 1e-5


def prepare(case, seed):
    s = {"case": case}
    m = _Make(seed)
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "checkpoint":
        s["x"] = m.activation(rows, cols, TYPES[case["type"]], case["pad"])
        s["scale"] = m.weight(cols) if case["affine"] else None
        s["shift"] = m.bias(cols) if case["affine"] else None
        return s
    if case["op"] == "weight_grad":
        s["dy"] = m.activation(rows, case["outs"], TYPES[case["type"]], case["pad"], 0.01)
        s["q"], s["e"] = _codes(m.activation(rows, cols, torch.float32))
        s["scale"] = m.weight(cols) if case["affine"] != "none" else None
        s["shift"] = m.bias(cols) if case["affine"] == "both" else None
        return s
    kind, stream = TYPES[case["type"]], TYPES[case["stream"]]
    for name in ("post", "pre"):
        used = case[name] != "none"
        s[name + "_weight"] = m.weight(cols) if used else None
        s[name + "_bias"] = m.bias(cols) if used and case["bias"] else None
    rpg = case["rows_per_gate"]
    s["gate"] = m.gate((rows + rpg - 1) // rpg, cols, TYPES[case["gate_type"]]) if rpg else None
    x = m.activation(rows, cols, stream, case["pad"], 2.0)
    f = m.activation(rows, cols, kind, case["pad"])
    if case["op"] == "edge":
        s["x"], s["f"] = x, f
        return s
    # what the forward pass left behind, and the gradients that arrive
    fh, f_mean, f_rstd = _norm(f.float(), case["post"], EPS)
    xh, x_mean, x_rstd = _norm(x.float(), case["pre"], EPS)
    zero = torch.zeros_like(x_mean)
    s["stats"] = torch.cat([zero if f_mean is None else f_mean, zero if f_rstd is None else f_rstd, x_mean, x_rstd], 1)
    if case["save"] == "checkpoint":
        s["post_q"], s["post_e"] = _codes(fh)
        s["pre_q"], s["pre_e"] = _codes(xh)
    else:
        s["f"], s["x_out"] = f, x
    s["dx_out"] = m.activation(rows, cols, stream, case["pad"], 0.01)
    s["du"] = m.activation(rows, cols, kind, case["pad"], 0.01)
    return s


# ----------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------

def _affine(v, weight, bias):
    if weight is not None:
        v = v * weight
    return v if bias is None else v + bias


def _gate_rows(s):
    """The gate of every row in fp32, or one."""
    if s["gate"] is None:
        return 1.0
    return s["gate"].float().repeat_interleave(s["case"]["rows_per_gate"], 0)[:s["case"]["rows"]]


def _plain_edge(s):
    case = s["case"]
    fh, f_mean, f_rstd = _norm(s["f"].float(), case["post"], EPS)
    branch = case["branch"] * _gate_rows(s) * _affine(fh, s["post_weight"], s["post_bias"])
    x = case["skip"] * s["x"].float() + branch
    xh, x_mean, x_rstd = _norm(x, case["pre"], EPS)
    out = {"x_out": x.to(s["x"].dtype), "u": _affine(xh, s["pre_weight"], s["pre_bias"]).to(s["f"].dtype)}
    if case["save"] == "checkpoint":
        zero = torch.zeros_like(x_mean)
        out["stats"] = torch.cat([zero if f_mean is None else f_mean, zero if f_rstd is None else f_rstd, x_mean, x_rstd], 1)
        out["post"] = _values(*_codes(fh)).to(torch.bfloat16)
        out["pre"] = _values(*_codes(xh)).to(torch.bfloat16)
    return out


def _norm_grad(dn, h, rstd, kind):
    """Gradient through a norm: dn at its normalised output h."""
    if kind == "none":
        return dn
    g = dn - h * (dn * h).mean(1, keepdim=True)
    if kind == "layer":
        g = g - dn.mean(1, keepdim=True)
    return g * rstd


def _plain_back(s):
    case = s["case"]
    f_mean, f_rstd, x_mean, x_rstd = s["stats"].split(1, 1)
    if case["save"] == "checkpoint":
        fh, xh = _values(s["post_q"], s["post_e"]), _values(s["pre_q"], s["pre_e"])
    else:
        fh = s["f"].float() if case["post"] == "none" else (s["f"].float() - f_mean) * f_rstd
        xh = (s["x_out"].float() - x_mean) * x_rstd
    du = s["du"].float()
    out = {"pre_weight": (du * xh).sum(0)}
    if s["pre_bias"] is not None:
        out["pre_bias"] = du.sum(0)
    d = s["dx_out"].float() + _norm_grad(du * s["pre_weight"], xh, x_rstd, case["pre"])
    out["dx"] = (case["skip"] * d).to(s["dx_out"].dtype)
    if s["gate"] is not None:
        rpg, rows, cols = case["rows_per_gate"], case["rows"], case["cols"]
        each = case["branch"] * d * _affine(fh, s["post_weight"], s["post_bias"])
        full = rows // rpg * rpg
        dgate = each[:full].view(-1, rpg, cols).sum(1)
        if full < rows:
            dgate = torch.cat([dgate, each[full:].sum(0, keepdim=True)])
        out["dgate"] = dgate.to(s["gate"].dtype)
    dn = case["branch"] * _gate_rows(s) * d
    if s["post_weight"] is not None:
        out["post_weight"] = (dn * fh).sum(0)
        dn_h = dn * s["post_weight"]
    else:
        dn_h = dn
    if s["post_bias"] is not None:
        out["post_bias"] = dn.sum(0)
    out["df"] = _norm_grad(dn_h, fh, f_rstd, case["post"]).to(s["du"].dtype)
    return out


def _plain_checkpoint(s):
    q, e = _codes(s["x"].float())
    return {"values": _values(q, e).to(torch.bfloat16),
            "out": _affine(_values(q, e), s["scale"], s["shift"]).to(s["x"].dtype)}


def _plain_grad(s):
    dy = s["dy"].float()
    out = {"dw": torch.matmul(dy.t(), _affine(_values(s["q"], s["e"]), s["scale"], s["shift"]))}
    if s["case"]["bias"]:
        out["db"] = dy.sum(0)
    return out


# ----------------------------------------------------------------------------
# the framework's operators
# ----------------------------------------------------------------------------

def _empty(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEVICE)


def _handle(s):
    """The layer's handle and the buffers for what it saves, which a program keeps from step to step."""
    from paper_1910_10929_amd import blocks
    case = s["case"]
    name = lambda kind: None if kind == "none" else kind  # noqa: E731
    s["edge"] = blocks.Edge(case["cols"], post=name(case["post"]), pre=name(case["pre"]), post_weight=s["post_weight"],
                            post_bias=s["post_bias"], pre_weight=s["pre_weight"], pre_bias=s["pre_bias"], eps=EPS,
                            skip_scale=case["skip"], branch_scale=case["branch"])
    if case["op"] == "edge":
        s["saved"] = blocks.Saved(case["rows"], case["cols"], device=DEVICE) if case["save"] == "checkpoint" else None
    elif case["save"] == "checkpoint":
        s["saved"] = blocks.Saved(case["rows"], case["cols"], stats=s["stats"],
                                  post=blocks.Checkpoint.of(s["post_q"], s["post_e"]),
                                  pre=blocks.Checkpoint.of(s["pre_q"], s["pre_e"]))
    else:
        s["saved"] = blocks.Saved(case["rows"], case["cols"], stats=s["stats"], f=s["f"], x_out=s["x_out"])


def _own_edge(s):
    if "edge" not in s:
        _handle(s)
    case, saved = s["case"], s["saved"]
    x_out, u = s["edge"].forward(s["x"], s["f"], gate=s["gate"], rows_per_gate=case["rows_per_gate"] or None, save=saved)
    out = {"x_out": x_out, "u": u}
    if saved is not None:
        out["stats"] = saved.stats
        out["post"] = saved.post.decode(dtype=torch.bfloat16)
        out["pre"] = saved.pre.decode(dtype=torch.bfloat16)
    return out


def _own_back(s):
    if "edge" not in s:
        _handle(s)
    case, cols = s["case"], s["case"]["cols"]
    out = {"pre_weight": _empty(cols)}
    for name in ("pre_bias", "post_weight", "post_bias"):
        if s[name] is not None:
            out[name] = _empty(cols)
    if s["gate"] is not None:
        out["dgate"] = torch.empty_like(s["gate"])
    out["dx"], out["df"] = s["edge"].backward(
        s["saved"], dx_out=s["dx_out"], du=s["du"], gate=s["gate"], rows_per_gate=case["rows_per_gate"] or None,
        dgate=out.get("dgate"), post_weight_grad=out.get("post_weight"), post_bias_grad=out.get("post_bias"),
        pre_weight_grad=out["pre_weight"], pre_bias_grad=out.get("pre_bias"))
    return out


def _own_checkpoint(s):
    from paper_1910_10929_amd import blocks
    c = blocks.Checkpoint(s["case"]["rows"], s["case"]["cols"], device=DEVICE)
    c.encode(s["x"])
    return {"values": c.decode(dtype=torch.bfloat16), "out": c.decode(dtype=s["x"].dtype, scale=s["scale"], shift=s["shift"])}


def _own_grad(s):
    from paper_1910_10929_amd import blocks
    case = s["case"]
    out = {"dw": _empty(case["outs"], case["cols"])}
    if case["bias"]:
        out["db"] = _empty(case["outs"])
    blocks.weight_grad(s["dy"], blocks.Checkpoint.of(s["q"], s["e"]), out["dw"], out.get("db"), scale=s["scale"],
                       shift=s["shift"])
    return out


_PLAIN = {"edge": _plain_edge, "edge_backward": _plain_back, "checkpoint": _plain_checkpoint, "weight_grad": _plain_grad}
_OWN = {"edge": _own_edge, "edge_backward": _own_back, "checkpoint": _own_checkpoint, "weight_grad": _own_grad}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------

def work(case):
    rows, cols = case["rows"], case["cols"]
    n, runs = rows * cols, rows * ((cols + RUN - 1) // RUN)
    if case["op"] == "checkpoint":
        b = BYTES[case["type"]]
        # (the codes are written and read again)
        return {"bytes": n * b + 2 * (n + runs) + 2 * n + b * n + (8 * cols if case["affine"] else 0), "flops": 8 * n}
    if case["op"] == "weight_grad":
        outs = case["outs"]
        vectors = {"none": 0, "scale": 1, "both": 2}[case["affine"]] * 4 * cols + (4 * outs if case["bias"] else 0)
        return {"bytes": rows * outs * BYTES[case["type"]] + n + runs + 4 * outs * cols + vectors, "flops": 2 * n * outs}
    b, x = BYTES[case["type"]], BYTES[case["stream"]]
    rpg = case["rows_per_gate"]
    gates = (rows + rpg - 1) // rpg * cols * BYTES[case["gate_type"]] if rpg else 0
    vectors = 4 * cols * ((case["post"] != "none") + (case["pre"] != "none")) * (2 if case["bias"] else 1)
    if case["op"] == "edge":
        saved = 2 * (n + runs) + 16 * rows + 2 * (n + runs) + 4 * n if case["save"] == "checkpoint" else 0
        return {"bytes": 2 * n * (x + b) + gates + vectors + saved, "flops": 20 * n}
    kept = 2 * (n + runs) if case["save"] == "checkpoint" else n * (x + b)
    return {"bytes": 2 * n * (x + b) + kept + 16 * rows + 2 * gates + 2 * vectors, "flops": 30 * n}


# ----------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------

def exact(case, seed):
    """From the definitions, in float64.  In the place of a checkpoint of computed values (the forward edge's) stand those
    values themselves: what is between two codes belongs to either, and the codes' distance from them is measured."""
    s = prepare(case, seed)
    D = torch.float64
    d = {k: v.to(D) for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    rows, cols = case["rows"], case["cols"]

    def read(q, e):
        power = torch.exp2(e.to(D) - 127.0)
        power[e == 255] = float("nan")
        wide = power[:, torch.arange(cols, device=DEVICE) // RUN]
        return wide.mul_(q)

    if case["op"] == "checkpoint":
        out = torch.empty((rows, cols), dtype=D, device=DEVICE)
        for lo in range(0, cols, RUN):
            part = d["x"][:, lo:lo + RUN]
            _, power = torch.frexp(part.abs().amax(1, keepdim=True))        # largest magnitude < 2^power
            step = torch.exp2((power - 7).clamp(-126, 121).to(D))
            step = torch.where((part.abs().amax(1, keepdim=True) >= 127.5 * step) & (power - 7 < 121), 2.0 * step, step)
            out[:, lo:lo + RUN] = (part / step).round_().clamp_(-127.0, 127.0).mul_(step)
        return {"values": out, "out": torch.addcmul(d["shift"], out, d["scale"]) if case["affine"] else out}
    if case["op"] == "weight_grad":
        u = read(s["q"], s["e"])
        if "scale" in d:
            u.mul_(d["scale"])
        if "shift" in d:
            u.add_(d["shift"])
        out = {"dw": (u.t() @ d["dy"]).t()}
        if case["bias"]:
            out["db"] = torch.ones(rows, dtype=D, device=DEVICE) @ d["dy"]
        return out
    rpg = case["rows_per_gate"]
    which = torch.arange(rows, device=DEVICE) // (rpg or 1)
    gate = d["gate"].index_select(0, which) if rpg else torch.ones((1, cols), dtype=D, device=DEVICE)
    one, none = torch.ones(cols, dtype=D, device=DEVICE), torch.zeros(cols, dtype=D, device=DEVICE)
    wp, bp = d.get("post_weight", one), d.get("post_bias", none)
    wn, bn = d["pre_weight"], d.get("pre_bias", none)

    def moments(v, kind):
        if kind == "none":
            return torch.zeros((rows, 1), dtype=D, device=DEVICE), torch.zeros((rows, 1), dtype=D, device=DEVICE)
        mean = v.sum(1, keepdim=True) / cols if kind == "layer" else torch.zeros((rows, 1), dtype=D, device=DEVICE)
        return mean, ((v - mean).square().sum(1, keepdim=True) / cols + EPS).sqrt().reciprocal()

    if case["op"] == "edge":
        fm, fr = moments(d["f"], case["post"])
        fh = d["f"] if case["post"] == "none" else (d["f"] - fm) * fr
        x = torch.addcmul(d["x"] * case["skip"], gate * case["branch"], fh * wp + bp)
        xm, xr = moments(x, case["pre"])
        xh = (x - xm) * xr
        out = {"x_out": x, "u": xh * wn + bn}
        if case["save"] == "checkpoint":
            out.update(stats=torch.cat([fm, fr, xm, xr], 1), post=fh, pre=xh)
        return out
    st = d["stats"]
    if case["save"] == "checkpoint":
        fh, xh = read(s["post_q"], s["post_e"]), read(s["pre_q"], s["pre_e"])
    else:
        fh = d["f"] if case["post"] == "none" else (d["f"] - st[:, 0:1]) * st[:, 1:2]
        xh = (d["x_out"] - st[:, 2:3]) * st[:, 3:4]

    def through(g, h, rstd, kind):
        # the projection that a norm's gradient is
        if kind == "none":
            return g
        out = g - (g * h).sum(1, keepdim=True) / cols * h
        return rstd * (out - g.sum(1, keepdim=True) / cols) if kind == "layer" else rstd * out

    delta = d["dx_out"] + through(d["du"] * wn, xh, st[:, 3:4], case["pre"])
    at_n = delta * gate * case["branch"]
    out = {"pre_weight": torch.linalg.vecdot(d["du"], xh, dim=0), "dx": delta * case["skip"],
           "df": through(at_n * wp, fh, st[:, 1:2], case["post"])}
    if s["pre_bias"] is not None:
        out["pre_bias"] = d["du"].sum(0)
    if s["post_weight"] is not None:
        out["post_weight"] = torch.linalg.vecdot(at_n, fh, dim=0)
    if s["post_bias"] is not None:
        out["post_bias"] = at_n.sum(0)
    if rpg:
        out["dgate"] = torch.zeros_like(d["gate"]).index_add_(0, which, delta * (fh * wp + bp) * case["branch"])
    return out
