"""Training blocks of libdgs: the binding of include/dgs_blocks.h.

The memory-bound part of a transformer worker's step, around `dgs.Context`: the edge between two blocks (norm of
the branch, gate, residual sum, norm of the stream) with its gradients, 8-bit checkpoints of activations, and the gradient of
a linear layer read from the checkpoint of its input; and the end of that step: the output layer with its loss and gradients,
and updates of weight matrices orthogonalised.  Parameters and their gradients are fp32 vectors and matrices -- slices
of the flat buffers that `dgs.Context` works on -- and gradients can be added to what is there.

Matrices are 2-d tensors whose columns are contiguous; rows may be any distance apart.  Work is enqueued on torch's
current stream of the tensors' device, and nothing waits.  What a call refuses, it refuses with `dgs.DgsError` before
anything is enqueued.  Nothing here is recorded by autograd.  There is no CPU fallback.
"""
from __future__ import annotations

import collections
import ctypes
import functools
import struct

import torch

from . import dgs
from .dgs import DGS_EINVAL, DGS_ENOTSUP, DgsError

F32, F16, BF16 = 0, 1, 2
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
EDGE_MAX_COLS = 16384
CHECKPOINT_RUN = 32
_MOST = 0x7FFFFFFF      # rows, or columns

EXPORTS = [
    "dgs_edge_forward", "dgs_edge_backward_workspace", "dgs_edge_backward", "dgs_checkpoint_encode", "dgs_checkpoint_decode",
    "dgs_checkpoint_weight_grad_workspace", "dgs_checkpoint_weight_grad", "dgs_head_workspace", "dgs_head_forward",
    "dgs_head_backward", "dgs_orthogonalise_workspace", "dgs_orthogonalise",
]

_TYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_NORMS = {None: NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}

# the argument structures of the header
_EDGE = struct.Struct("@Iii4f4P")
_FORWARD = struct.Struct("@II4i" + "PQ" * 5 + "PQPQ" * 2 + "P")
_BACKWARD = struct.Struct("@II4i" + "PQ" * 5 + "PQPQ" * 2 + "P" + "PQ" * 3 + "4P" + "PQ")
_CODES = struct.Struct("@PQPQ")
_GRAD = struct.Struct("@III3i" + "PQ" + "PQPQ" + "PP" + "PQ" + "P" + "PQ")
_HEAD = struct.Struct("@III3i" + "PQ" * 2 + "PP" + "PP" + "PP" + "PQ" + "PQ" + "P" + "PQ")
_ORTHOGONALISE = struct.Struct("@IIII4i5f" + "PP" + "PQ")

_lib = None


def lib():
    global _lib
    if _lib is None:
        L = dgs.lib()
        vp, u32, u64, i32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int
        L.dgs_edge_forward.argtypes = [vp, vp, vp]
        L.dgs_edge_backward_workspace.restype = ctypes.c_size_t
        L.dgs_edge_backward_workspace.argtypes = [u32, u32, u32]
        L.dgs_edge_backward.argtypes = [vp, vp, vp]
        L.dgs_checkpoint_encode.argtypes = [u32, u32, i32, vp, u64, vp, vp]
        L.dgs_checkpoint_decode.argtypes = [u32, u32, vp, vp, vp, i32, vp, u64, vp]
        L.dgs_checkpoint_weight_grad_workspace.restype = ctypes.c_size_t
        L.dgs_checkpoint_weight_grad_workspace.argtypes = [u32, u32, u32, i32]
        L.dgs_checkpoint_weight_grad.argtypes = [vp, vp]
        L.dgs_head_workspace.restype = ctypes.c_size_t
        L.dgs_head_workspace.argtypes = [vp, i32]
        L.dgs_head_forward.argtypes = [vp, vp]
        L.dgs_head_backward.argtypes = [vp, vp]
        L.dgs_orthogonalise_workspace.restype = ctypes.c_size_t
        L.dgs_orthogonalise_workspace.argtypes = [vp]
        L.dgs_orthogonalise.argtypes = [vp, vp]
        _lib = L
    return _lib


def _refuse(what):
    raise DgsError(DGS_EINVAL, what)


def _fits(n, what):
    """(Sizes go to the library in 32 bits, and would arrive as what is left of them.)"""
    if n > _MOST:
        raise DgsError(DGS_ENOTSUP, f"{what}: more than 2^31 - 1")


def _type(t, what):
    k = _TYPES.get(t.dtype)
    if k is None:
        _refuse(f"{what}: {t.dtype} is not supported")
    return k


def _on_gpu(t, what):
    device = t.get_device()
    if device < 0:
        _refuse(f"{what} is not on a GPU")
    return device


def _matrix(t, rows, cols, device, what):
    """Pointer and stride of a rows x cols matrix on `device`."""
    if t.shape != (rows, cols):
        _refuse(f"{what}: shape {tuple(t.shape)}, expected ({rows}, {cols})")
    if t.get_device() != device:
        _refuse(f"{what} is on another device")
    stride, unit = t.stride()
    if unit != 1 and cols > 1:
        _refuse(f"{what}: columns are not contiguous")
    if stride < cols:
        if rows > 1:
            _refuse(f"{what}: rows overlap")
        stride = cols
    return t.data_ptr(), stride


def _vector(t, n, device, what):
    """Pointer of n contiguous floats on `device`, 0 for none."""
    if t is None:
        return 0
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        _refuse(f"{what}: expected {n} contiguous float32 values")
    if t.get_device() != device:
        _refuse(f"{what} is on another device")
    return t.data_ptr()


# the handle of torch's current stream of a device, and the current device (the short way is a fifth of a small call's time shorter)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _enqueue(what, device, call, *args):
    """call(*args, stream) on torch's current stream of the device."""
    if _current_device() == device:
        rc = call(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            rc = call(*args, _raw_stream(device))
    if rc:
        raise DgsError(rc, what)


@functools.lru_cache(maxsize=1024)
def _backward_bytes(rows, cols, rows_per_gate):
    return lib().dgs_edge_backward_workspace(rows, cols, rows_per_gate)


@functools.lru_cache(maxsize=1024)
def _weight_grad_bytes(rows, outs, cols, kind):
    return lib().dgs_checkpoint_weight_grad_workspace(rows, outs, cols, kind)


def _like(t, dtype, cols):
    """A new matrix of the shape of `t`, whose columns are contiguous, with its pointer and stride."""
    new = torch.empty_like(t, dtype=dtype)
    return new, (new.data_ptr(), cols)


def _workspace(given, need, like, device, what):
    if given is None:
        return like.new_empty(max(need, 16), dtype=torch.uint8)
    if given.get_device() != device or not given.is_contiguous():
        _refuse(f"{what}: workspace is not contiguous memory of the device")
    return given


class Checkpoint:
    """A rows x cols matrix in 8 bits: `codes` (int8) and `exps` (uint8, one for 32 columns of a row)."""

    def __init__(self, rows, cols, device="cuda:0", codes=None, exps=None):
        _fits(rows, "rows")
        _fits(cols, "columns")
        self.rows, self.cols = rows, cols
        runs = self._runs = (cols + CHECKPOINT_RUN - 1) // CHECKPOINT_RUN
        if codes is None and exps is None:
            codes = torch.empty((rows, cols), dtype=torch.int8, device=device)
            self.codes, self.exps = codes, codes.new_empty((rows, runs), dtype=torch.uint8)
            _on_gpu(codes, "checkpoint")
            return
        if codes is None or exps is None or codes.dtype != torch.int8 or exps.dtype != torch.uint8:
            _refuse("a checkpoint's codes are int8 and its exponents uint8")
        self.codes, self.exps = codes, exps
        device = _on_gpu(codes, "checkpoint")
        _matrix(codes, rows, cols, device, "codes")
        _matrix(exps, rows, runs, device, "exps")

    @classmethod
    def of(cls, codes, exps):
        """A checkpoint that lies in the given tensors."""
        if codes.dim() != 2:
            _refuse("codes: expected a matrix")
        return cls(codes.shape[0], codes.shape[1], codes=codes, exps=exps)

    def _place(self, rows, cols, device, what):
        if self.rows != rows or self.cols != cols:
            _refuse(f"{what}: a checkpoint of ({self.rows}, {self.cols}), expected ({rows}, {cols})")
        codes, exps = self.codes, self.exps
        if codes.get_device() != device:
            _refuse(f"{what} is on another device")
        # (one row: any stride will do)
        return codes.data_ptr(), max(codes.stride(0), cols), exps.data_ptr(), max(exps.stride(0), self._runs)

    def encode(self, x):
        """Hold x from now on."""
        device = _on_gpu(x, "x")
        data, stride = _matrix(x, self.rows, self.cols, device, "x")
        _enqueue("dgs_checkpoint_encode", device, lib().dgs_checkpoint_encode, self.rows, self.cols, _type(x, "x"), data, stride,
                 _CODES.pack(*self._place(self.rows, self.cols, device, "checkpoint")))
        return self

    def decode(self, out=None, dtype=torch.float32, scale=None, shift=None):
        """The values, times `scale` and plus `shift` (fp32, one for each column), in `out` or a new tensor of `dtype`."""
        device = self.codes.get_device()
        if out is None:
            out, (data, stride) = _like(self.codes, dtype, self.cols)
        else:
            data, stride = _matrix(out, self.rows, self.cols, device, "out")
        _enqueue("dgs_checkpoint_decode", device, lib().dgs_checkpoint_decode, self.rows, self.cols,
                 _CODES.pack(*self._place(self.rows, self.cols, device, "checkpoint")),
                 _vector(scale, self.cols, device, "scale"), _vector(shift, self.cols, device, "shift"), _type(out, "out"), data,
                 stride)
        return out


class Saved:
    """What `Edge.forward` keeps of `rows` rows for `Edge.backward`: the norms' statistics, and of each norm's result a
    checkpoint (`post`, `pre`) or, with checkpoints=False, the matrices it was taken of (`f`, `x_out`), by reference: those must
    stay as they are until then.  `branch`: whether there was one; without a forward pass (None), whether something of it is
    here.  `dtypes`: the stream's and the branch's."""

    def __init__(self, rows, cols, device="cuda:0", checkpoints=True, stats=None, post=None, pre=None, f=None, x_out=None):
        _fits(rows, "rows")
        given = post is not None or pre is not None or f is not None or x_out is not None
        self.rows, self.cols = rows, cols
        self.stats = stats if stats is not None else torch.empty((rows, 4), dtype=torch.float32, device=device)
        self.post, self.pre, self.f, self.x_out = post, pre, f, x_out
        self.branch, self.dtypes = None, (None, None)
        if checkpoints and not given:
            self.post, self.pre = Checkpoint(rows, cols, device), Checkpoint(rows, cols, device)


_NO_MATRIX = (0, 0)
_NO_CODES = (0, 0, 0, 0)


class Edge:
    """The edge between two blocks of a model of `cols` channels; see dgs_edge in the header.

        x_out = skip_scale * x + branch_scale * gate * (N_post(f) * post_weight + post_bias)
        u     = N_pre(x_out) * pre_weight + pre_bias

    post, pre: "rms", "layer" or None; weights and biases: fp32 vectors or None (1 and 0)."""

    def __init__(self, cols, post=None, pre=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None, eps=1e-5,
                 post_eps=None, pre_eps=None, skip_scale=1.0, branch_scale=1.0):
        if post not in _NORMS or pre not in _NORMS:
            _refuse("post and pre are 'rms', 'layer' or None")
        if post is None and (post_weight is not None or post_bias is not None):
            _refuse("post_weight and post_bias need a norm")
        if pre is None and (pre_weight is not None or pre_bias is not None):
            _refuse("pre_weight and pre_bias need a norm")
        _fits(cols, "columns")
        self.cols, self.post, self.pre = cols, post, pre
        self._fixed = (cols, _NORMS[post], _NORMS[pre], eps if post_eps is None else post_eps, eps if pre_eps is None else pre_eps,
                       skip_scale, branch_scale)
        vectors = {"post_weight": post_weight, "post_bias": post_bias, "pre_weight": pre_weight, "pre_bias": pre_bias}
        self._vectors = tuple(vectors.values())
        self._device = None
        for name, v in vectors.items():
            if v is not None:
                self._device = _on_gpu(v, name) if self._device is None else self._device
                _vector(v, cols, self._device, name)

    # (fixed when the edge is made)
    post_weight = property(lambda self: self._vectors[0])
    post_bias = property(lambda self: self._vectors[1])
    pre_weight = property(lambda self: self._vectors[2])
    pre_bias = property(lambda self: self._vectors[3])

    def _layer(self, device):
        if self._device is not None and self._device != device:
            _refuse("the edge's parameters are on another device")
        return _EDGE.pack(*self._fixed, *[0 if v is None else v.data_ptr() for v in self._vectors])

    def _gate(self, gate, rows_per_gate, rows, device):
        """Pointer and stride, type, rows for each gate row."""
        if gate is None:
            return _NO_MATRIX, F32, 0
        if gate.dim() != 2:
            _refuse("gate: expected a matrix")
        count = gate.shape[0]
        if rows_per_gate is None:
            if rows and (count == 0 or rows % count):
                _refuse("gate: rows_per_gate is needed where the gate rows do not divide the rows")
            rows_per_gate = max(rows // count, 1) if rows else 1
        elif rows_per_gate < 1:
            _refuse("rows_per_gate is at least 1")
        if rows:      # (any gate goes with no rows)
            count = (rows + rows_per_gate - 1) // rows_per_gate
        return _matrix(gate, count, self.cols, device, "gate"), _type(gate, "gate"), min(rows_per_gate, _MOST)

    def forward(self, x, f=None, gate=None, rows_per_gate=None, x_out=None, u=None, save=None):
        """One pass over the rows; returns (x_out, u).  Without f there is no branch: x_out is x.  Without `pre`, u is None.
        x_out may be x, and u may be f unless `save` keeps f itself.  save: a `Saved` that is filled."""
        device = _on_gpu(x, "x")
        if x.dim() != 2:
            _refuse("x: expected a matrix")
        rows, cols = x.size(0), self.cols
        _fits(rows, "rows")
        px = _matrix(x, rows, cols, device, "x")
        stream = _type(x, "x")
        pf = pg = po = pu = _NO_MATRIX
        gate_type, per = F32, 0
        kind = stream
        if f is not None:
            pf, kind = _matrix(f, rows, cols, device, "f"), _type(f, "f")
            pg, gate_type, per = self._gate(gate, rows_per_gate, rows, device)
            if x_out is None:
                x_out, po = _like(x, x.dtype, cols)
            elif x_out.dtype != x.dtype:
                _refuse("x_out: expected the type of x")
            else:
                po = _matrix(x_out, rows, cols, device, "x_out")
        elif gate is not None or x_out is not None:
            _refuse("without f there is no gate and no x_out")
        if self.pre is not None:
            if u is None:
                u, pu = _like(x, x.dtype, cols) if f is None else _like(f, f.dtype, cols)
            elif f is not None and u.dtype != f.dtype:
                _refuse("u: expected the type of f")
            else:
                kind, pu = _type(u, "u"), _matrix(u, rows, cols, device, "u")
        elif u is not None:
            _refuse("u needs a norm before the block")
        post = pre = _NO_CODES
        stats = 0
        if save is not None:
            if save.rows != rows or save.cols != cols:
                _refuse("save: of another shape")
            stats = _vector(save.stats, 4 * rows, device, "stats")
            if f is not None and save.post is not None:
                post = save.post._place(rows, cols, device, "save.post")
            if self.pre is not None and save.pre is not None:
                pre = save.pre._place(rows, cols, device, "save.pre")
            # (a tensor without memory is at 0, and so is one that is not there)
            if (save.post is None and pf[0] and pf[0] in (po[0], pu[0])) or (save.pre is None and pu[0] and pu[0] == (px if f is None else po)[0]):
                _refuse("save: an output lies over a matrix that is kept for the backward pass")
        _enqueue("dgs_edge_forward", device, lib().dgs_edge_forward, self._layer(device),
                 _FORWARD.pack(rows, per, stream, kind, gate_type, 0, *px, *pf, *pg, *po, *pu, *post, *pre, stats))
        if save is not None:
            save.branch, save.dtypes = f is not None, (x.dtype, f.dtype if f is not None else u.dtype)
            if save.post is None:
                save.f = f
            if save.pre is None:
                save.x_out = x if f is None else x_out
        return (x if f is None else x_out), u

    def backward(self, saved, dx_out=None, du=None, gate=None, rows_per_gate=None, dx=None, df=None, dgate=None,
                 post_weight_grad=None, post_bias_grad=None, pre_weight_grad=None, pre_bias_grad=None, accumulate=False,
                 workspace=None):
        """Gradients, from those that arrive at x_out and u (None: zero); returns (dx, df), df None for an edge without a
        branch.  Parameter gradients are written, or with `accumulate` added, to the fp32 vectors given; dgate (gate's type)
        is written, or added to where it is fp32.  dx may be dx_out, df may be du; new ones have the types of dx_out and du, or
        where those are absent of x and f."""
        given = dx_out if dx_out is not None else du
        if given is None:
            _refuse("dx_out or du is needed")
        device = _on_gpu(given, "gradient")
        rows, cols = saved.rows, self.cols
        if saved.cols != cols:
            _refuse("saved: of another shape")
        coded = saved.post is not None
        branch = coded or saved.f is not None
        if saved.branch is not None:
            if saved.branch and not branch:
                _refuse("saved: nothing of the branch")
            branch = saved.branch
        pd = pu = pf = px = pdf = pdg = _NO_MATRIX
        post = pre = _NO_CODES
        stream_dtype = (dx_out.dtype if dx_out is not None else saved.x_out.dtype if saved.x_out is not None else
                        dx.dtype if dx is not None else None)
        dtype = (du.dtype if du is not None else saved.f.dtype if saved.f is not None else df.dtype if df is not None else None)
        # A type that nothing given says is that of the forward pass, where that goes with the other type, and otherwise the other.
        if stream_dtype is None:
            kept = saved.dtypes[0]
            stream_dtype = kept if kept in (torch.float32, dtype) else dtype
        if dtype is None:
            kept = saved.dtypes[1]
            dtype = kept if kept is not None and stream_dtype in (torch.float32, kept) else stream_dtype
        if dx_out is not None:
            pd = _matrix(dx_out, rows, cols, device, "dx_out")
        if du is not None:
            if self.pre is None:
                _refuse("du needs a norm before the block")
            pu = _matrix(du, rows, cols, device, "du")
            if branch and coded != (saved.pre is not None):
                _refuse("saved: both norms as checkpoints or both as values")
            if saved.pre is not None:
                pre = saved.pre._place(rows, cols, device, "saved.pre")
            elif saved.x_out is None:
                _refuse("saved: nothing of the norm before the block")
            else:
                px = _matrix(saved.x_out, rows, cols, device, "saved.x_out")
                if saved.x_out.dtype != stream_dtype:
                    _refuse("saved.x_out: expected the type of dx_out")
        if branch:
            if coded:
                post = saved.post._place(rows, cols, device, "saved.post")
            else:
                pf = _matrix(saved.f, rows, cols, device, "saved.f")
                if saved.f.dtype != dtype:
                    _refuse("saved.f: expected the type of du")
            if df is None:
                df, pdf = _like(given, dtype, cols)
            elif df.dtype != dtype:
                _refuse("df: expected the type of du")
            else:
                pdf = _matrix(df, rows, cols, device, "df")
        elif df is not None:
            _refuse("df: the edge has no branch")
        pg, gate_type, per = self._gate(gate, rows_per_gate, rows, device)
        if dgate is not None:
            if gate is None or dgate.dtype != gate.dtype:
                _refuse("dgate: expected a gate of the same type")
            pdg = _matrix(dgate, gate.shape[0], cols, device, "dgate")
        if dx is None:
            dx, pdx = _like(given, stream_dtype, cols)
        elif dx.dtype != stream_dtype:
            _refuse("dx: expected the type of dx_out")
        else:
            pdx = _matrix(dx, rows, cols, device, "dx")
        grads = (_vector(post_weight_grad, cols, device, "post_weight_grad"), _vector(post_bias_grad, cols, device, "post_bias_grad"),
                 _vector(pre_weight_grad, cols, device, "pre_weight_grad"), _vector(pre_bias_grad, cols, device, "pre_bias_grad"))
        ws = _workspace(workspace, _backward_bytes(rows, cols, per), given, device, "dgs_edge_backward")
        _enqueue("dgs_edge_backward", device, lib().dgs_edge_backward, self._layer(device),
                 _BACKWARD.pack(rows, per, _TYPES.get(stream_dtype, -1), _TYPES.get(dtype, -1), gate_type, int(accumulate), *pd, *pu,
                                *pg, *pf, *px, *post, *pre, _vector(saved.stats, 4 * rows, device, "stats"), *pdx, *pdf, *pdg,
                                *grads, ws.data_ptr(), ws.numel() * ws.element_size()))
        if rows == 0 and dgate is not None and not (accumulate and dgate.dtype == torch.float32):
            dgate.zero_()       # (the library knows of no gate rows then)
        return dx, df


def weight_grad(dy, saved, dw, db=None, scale=None, shift=None, accumulate=False, workspace=None):
    """Gradient of y = u W^T + b, u being the values of the checkpoint `saved` times `scale` plus `shift`: dw = dy^T u
    (outs x cols, fp32, may have any distance between rows) and db = the sum of dy's rows; with `accumulate` added."""
    device = _on_gpu(dy, "dy")
    if dy.dim() != 2 or dw.dim() != 2:
        _refuse("dy and dw: expected matrices")
    rows, outs, cols = dy.shape[0], dy.shape[1], saved.cols
    _fits(outs, "outputs")
    if dw.dtype != torch.float32:
        _refuse("dw: expected float32")
    kind = _type(dy, "dy")
    ws = _workspace(workspace, _weight_grad_bytes(rows, outs, cols, kind), dy, device, "dgs_checkpoint_weight_grad")
    _enqueue("dgs_checkpoint_weight_grad", device, lib().dgs_checkpoint_weight_grad,
             _GRAD.pack(rows, outs, cols, kind, int(accumulate), 0, *_matrix(dy, rows, outs, device, "dy"),
                        *saved._place(rows, cols, device, "saved"), _vector(scale, cols, device, "scale"),
                        _vector(shift, cols, device, "shift"), *_matrix(dw, outs, cols, device, "dw"),
                        _vector(db, outs, device, "db"), ws.data_ptr(), ws.numel() * ws.element_size()))
    return dw


_TARGETS = {torch.int64: 8, torch.int32: 4}


class Head:
    """The output layer with its loss, of which no logits are kept; see dgs_head_args in the header.

        z = x W^T + bias,   lse_t = log sum_v exp z_tv,   loss_t = lse_t - z_t[target_t]

    weight: vocab x cols, of the type that x has; bias: an fp32 vector or None.  Both are read when a call runs, so they may be
    updated in place between two steps.  A row whose target is no entry of the vocabulary (negative: padding) is left out."""

    def __init__(self, weight, bias=None):
        if weight.dim() != 2:
            _refuse("weight: expected a matrix")
        self.vocab, self.cols = weight.shape
        if self.vocab == 0 or self.cols == 0:
            _refuse("weight: no entries or no columns")
        _fits(self.vocab, "entries")
        _fits(self.cols, "columns")
        self._device = _on_gpu(weight, "weight")
        _type(weight, "weight")
        _matrix(weight, self.vocab, self.cols, self._device, "weight")
        _vector(bias, self.vocab, self._device, "bias")
        self.weight, self.bias = weight, bias

    def _rows(self, x, targets):
        device = _on_gpu(x, "x")
        if x.dim() != 2:
            _refuse("x: expected a matrix")
        if device != self._device:
            _refuse("the weight is on another device")
        if x.dtype != self.weight.dtype:
            _refuse("x: expected the type of the weight")
        rows = x.size(0)
        _fits(rows, "rows")
        size = _TARGETS.get(targets.dtype)
        if size is None or targets.numel() != rows or not targets.is_contiguous():
            _refuse(f"targets: expected {rows} contiguous int64 or int32 values")
        if targets.get_device() != device:
            _refuse("targets are on another device")
        return device, rows, size

    def _call(self, what, call, backward, device, rows, size, accumulate, x, targets, loss, lse, dloss, dlse, dx, dweight, dbias, workspace):
        fixed = (rows, self.cols, self.vocab, _TYPES[x.dtype], size, int(accumulate), *_matrix(x, rows, self.cols, device, "x"),
                 *_matrix(self.weight, self.vocab, self.cols, device, "weight"), _vector(self.bias, self.vocab, device, "bias"),
                 targets.data_ptr(), _vector(loss, rows, device, "loss"), _vector(lse, rows, device, "lse"),
                 _vector(dloss, rows, device, "dloss"), _vector(dlse, rows, device, "dlse"), *dx, *dweight, dbias)
        need = lib().dgs_head_workspace(_HEAD.pack(*fixed, 0, 0), backward)
        ws = _workspace(workspace, need, x, device, what)
        _enqueue(what, device, call, _HEAD.pack(*fixed, ws.data_ptr(), ws.numel() * ws.element_size()))

    def forward(self, x, targets, loss=None, lse=None, workspace=None):
        """(loss, lse), fp32, one for each row of x; targets: int64 or int32."""
        device, rows, size = self._rows(x, targets)
        if loss is None:
            loss = x.new_empty(rows, dtype=torch.float32)
        if lse is None:
            lse = x.new_empty(rows, dtype=torch.float32)
        self._call("dgs_head_forward", lib().dgs_head_forward, 0, device, rows, size, False, x, targets, loss, lse, None, None, _NO_MATRIX,
                   _NO_MATRIX, 0, workspace)
        return loss, lse

    def backward(self, x, targets, lse, dloss=None, dlse=None, dx=None, dweight=None, dbias=None, need_dx=True, accumulate=False,
                 workspace=None):
        """Gradients, from those that arrive at loss (None: 1) and lse (None: 0), fp32 vectors; x, targets and lse as in the forward
        pass.  Returns dx (None without need_dx); dweight (vocab x cols, fp32, may have any distance between rows) and dbias (fp32) are
        written, or with `accumulate` added to, where they are given."""
        device, rows, size = self._rows(x, targets)
        pdx = pdw = _NO_MATRIX
        if dx is not None:
            if dx.dtype != x.dtype:
                _refuse("dx: expected the type of x")
            if not need_dx:
                _refuse("dx is given and not needed")
            pdx = _matrix(dx, rows, self.cols, device, "dx")
            if dx.data_ptr() == x.data_ptr() and rows:
                _refuse("dx lies over x")
        elif need_dx:
            dx, pdx = _like(x, x.dtype, self.cols)
        if dweight is not None:
            if dweight.dtype != torch.float32:
                _refuse("dweight: expected float32")
            pdw = _matrix(dweight, self.vocab, self.cols, device, "dweight")
            if dweight.data_ptr() == self.weight.data_ptr():
                _refuse("dweight lies over the weight")
        if lse is None:
            _refuse("lse: the forward pass's is needed")
        self._call("dgs_head_backward", lib().dgs_head_backward, 1, device, rows, size, accumulate, x, targets, None, lse, dloss, dlse, pdx,
                   pdw, _vector(dbias, self.vocab, device, "dbias"), workspace)
        return dx


def orthogonalise(updates, out=None, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, scale=1.0, accumulate=False,
                  workspace=None):
    """Updates of weight matrices -- one matrix, or a list of matrices of one shape and type -- with their singular vectors kept
    and their singular values taken near 1 by Newton-Schulz products; see dgs_orthogonalise in the header.  Of each: X = G / (|G| + eps),
    `steps` times X = a X + (b A + c A^2) X with A = X X^T (of the smaller side), then out = scale X, or with `accumulate` out + scale X.
    `out`: as `updates`, of any one of the three types, or new ones of the updates' type; each may be its own update.  fp32 and half
    results take 22 bits of the operands to the products, bfloat16 ones 11."""
    one = isinstance(updates, torch.Tensor)
    given = [updates] if one else list(updates)
    if not given:
        return []
    if out is None:
        if accumulate:
            _refuse("out: nothing to add to")
        outs = None
    else:
        outs = [out] if isinstance(out, torch.Tensor) else list(out)
        if len(outs) != len(given) or one != isinstance(out, torch.Tensor):
            _refuse("out: expected as many matrices as updates")
    first = given[0]
    device = _on_gpu(first, "updates")
    if first.dim() != 2:
        _refuse("updates: expected matrices")
    rows, cols = first.shape
    if rows == 0 or cols == 0:
        _refuse("updates: no rows or no columns")
    _fits(rows, "rows")
    _fits(cols, "columns")
    kind = _type(first, "updates")
    if outs is None:
        outs = [torch.empty((rows, cols), dtype=first.dtype, device=first.device) for _ in given]
    out_kind = _type(outs[0], "out")
    if not isinstance(steps, int) or not 1 <= steps <= 1000 or len(coefficients) != 3:
        _refuse("steps: 1 to 1000; coefficients: three")
    places, out_places = [], []
    for g, o in zip(given, outs):
        if g.dtype != first.dtype or o.dtype != outs[0].dtype:
            _refuse("updates, and out: expected one type each")
        places += _matrix(g, rows, cols, device, "updates")
        out_places += _matrix(o, rows, cols, device, "out")
    if len(set(out_places[::2])) != len(outs):
        _refuse("out: one matrix twice")
    given_at = collections.Counter(places[::2])
    if any(given_at[o] > (o == i) for i, o in zip(places[::2], out_places[::2])):
        _refuse("out: lies over another update than its own")
    table = struct.pack(f"@{2 * len(places)}Q", *places, *out_places)
    table = ctypes.create_string_buffer(table, len(table))
    at = ctypes.addressof(table)
    fixed = (len(given), rows, cols, steps, kind, out_kind, int(accumulate), 0, *coefficients, eps, scale, at, at + 8 * len(places))
    need = lib().dgs_orthogonalise_workspace(_ORTHOGONALISE.pack(*fixed, 0, 0))
    ws = _workspace(workspace, need, first, device, "dgs_orthogonalise")
    _enqueue("dgs_orthogonalise", device, lib().dgs_orthogonalise, _ORTHOGONALISE.pack(*fixed, ws.data_ptr(), ws.numel() * ws.element_size()))
    return outs[0] if one else outs
