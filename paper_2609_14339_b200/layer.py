"""The layer around the step: layer norm, linear layers and activations kept in 8 bits, as functions on CUDA tensors.

Same conventions as the rest of the binding: argument marshalling only, every arithmetic step runs in the library's
kernels, work is queued on `stream` (default: the current stream) and nothing waits for it. Matrices are 2-D tensors
whose columns are contiguous; their rows may be apart (a slice of a wider buffer). What a call allocates (outputs not
passed in, workspaces) comes from the pool of the stream the work is queued on, so it is safe to let go of at once.
"""
from __future__ import annotations

import torch

from .binding import (SC_ACT_GELU, SC_ACT_NONE, SC_ACT_RELU, SC_ACT_SILU, SC_DTYPE_BF16, SC_DTYPE_FP32, SCError, _check,
                      load_library)

ACTIVATIONS = {"none": SC_ACT_NONE, "relu": SC_ACT_RELU, "gelu": SC_ACT_GELU, "silu": SC_ACT_SILU}
_DTYPES = {torch.bfloat16: SC_DTYPE_BF16, torch.float32: SC_DTYPE_FP32}


class _Queue:
    """The device and stream of one call: allocations come from that stream's pool, the launch goes to it."""

    def __init__(self, tensor, stream):
        self.device = tensor.device
        current = torch.cuda.current_stream(self.device)
        self.stream = current if stream is None else stream
        here = self.device.index == torch.cuda.current_device()
        self._guard = None if here and self.stream == current else torch.cuda.stream(self.stream)

    def __enter__(self):
        if self._guard is not None:
            self._guard.__enter__()
        return self

    def __exit__(self, *exc):
        if self._guard is not None:
            self._guard.__exit__(*exc)

    def empty(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)


def _act(act) -> int:
    if act not in ACTIVATIONS:
        raise ValueError("act must be one of %s, got %r" % (", ".join(sorted(ACTIVATIONS)), act))
    return ACTIVATIONS[act]


def _matrix(name, t, shape=None, dtype=None, device=None):
    """Row stride of a matrix argument, after its checks."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 2:
        raise ValueError("%s must be a 2-D CUDA tensor" % name)
    if t.dtype not in _DTYPES or (dtype is not None and t.dtype != dtype):
        raise ValueError("%s has dtype %s, expected %s" % (name, t.dtype, dtype if dtype is not None else "bfloat16 or float32"))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError("%s: columns must be contiguous" % name)
    if rows <= 1:
        return cols
    if t.stride(0) < cols:
        raise ValueError("%s: rows overlap" % name)
    return t.stride(0)


def _vector(name, t, n, device):
    if t is None:
        return None
    if not t.is_cuda or t.device != device or t.dtype != torch.float32 or tuple(t.shape) != (n,) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous float32 tensor of shape (%d,) on %s" % (name, n, device))
    return t.data_ptr()


def _status(t, device):
    if t is None:
        return None
    if not t.is_cuda or t.device != device or t.element_size() != 4 or t.numel() < 1:
        raise ValueError("status must be a 32-bit tensor on %s" % device)
    return t.data_ptr()


def _buffer(name, t, need, device):
    if t.dtype != torch.uint8 or not t.is_cuda or t.device != device or not t.is_contiguous() or t.numel() < need:
        raise ValueError("%s must be a contiguous uint8 tensor of at least %d bytes on %s" % (name, need, device))
    return t.data_ptr()


def _ptr(t):
    return None if t is None else t.data_ptr()


class Act8:
    """An activation kept in 8 bits: blocks of 32 features share a power of two (33 bytes for 32 values)."""

    def __init__(self, tokens: int, features: int, data):
        need = load_library().sc_act8_bytes(int(tokens), int(features))
        if need == 0:
            raise SCError(-2, "sc_act8_bytes")
        _buffer("data", data, need, data.device)
        self.tokens, self.features, self.data = int(tokens), int(features), data

    @classmethod
    def empty(cls, tokens: int, features: int, device="cuda:0") -> "Act8":
        return cls(tokens, features, torch.empty(cls.nbytes(tokens, features), dtype=torch.uint8, device=device))

    @staticmethod
    def nbytes(tokens: int, features: int) -> int:
        need = load_library().sc_act8_bytes(int(tokens), int(features))
        if need == 0:
            raise SCError(-2, "sc_act8_bytes")
        return int(need)


def _saved(name, saved, tokens, features, device):
    if saved is None:
        return None
    if not isinstance(saved, Act8):
        raise ValueError("%s must be an Act8" % name)
    if (saved.tokens, saved.features) != (tokens, features) or saved.data.device != device:
        raise ValueError("%s holds %d x %d on %s, expected %d x %d on %s" % (name, saved.tokens, saved.features,
                                                                            saved.data.device, tokens, features, device))
    return saved.data.data_ptr()


def layer_norm(X, weight=None, bias=None, eps: float = 1e-5, save=None, out=None, stats=None, stream=None):
    """Y = (X - mean) * rstd * weight + bias over each row. Returns (Y, stats); stats (2 x rows fp32: means, rstds) is
    what layer_norm_backward takes. save: an Act8 of X's shape that receives Y in 8 bits. out may be X."""
    ldx = _matrix("X", X)
    rows, cols = X.shape
    dev = X.device
    w, b = _vector("weight", weight, cols, dev), _vector("bias", bias, cols, dev)
    a8 = _saved("save", save, rows, cols, dev)
    with _Queue(X, stream) as q:
        out = q.empty((rows, cols), X.dtype) if out is None else out
        stats = q.empty((2, rows), torch.float32) if stats is None else stats
        if stats.dtype != torch.float32 or stats.numel() != 2 * rows or not stats.is_contiguous() or stats.device != dev:
            raise ValueError("stats must be a contiguous float32 tensor of 2 x %d values on %s" % (rows, dev))
        ldy = _matrix("out", out, (rows, cols), X.dtype, dev)
        _check(load_library().sc_layernorm_forward(X.data_ptr(), _DTYPES[X.dtype], w, b, float(eps), out.data_ptr(),
                                                   stats.data_ptr(), a8, rows, cols, ldx, ldy, q.stream.cuda_stream),
               "sc_layernorm_forward")
    return out, stats


def layer_norm_backward(dY, X, weight, stats, residual_grad=None, out=None, dweight=None, dbias=None, workspace=None,
                        stream=None):
    """(dX, dweight, dbias) of layer_norm; residual_grad (the gradient that reaches X around the block) is added to dX.
    out may be dY or residual_grad. workspace: uint8, sc_layernorm_workspace_bytes(rows, cols)."""
    ldx = _matrix("X", X)
    rows, cols = X.shape
    dev = X.device
    lddy = _matrix("dY", dY, (rows, cols), X.dtype, dev)
    ldr = _matrix("residual_grad", residual_grad, (rows, cols), X.dtype, dev) if residual_grad is not None else 0
    w = _vector("weight", weight, cols, dev)
    if stats.dtype != torch.float32 or stats.numel() != 2 * rows or not stats.is_contiguous() or stats.device != dev:
        raise ValueError("stats must be the contiguous float32 tensor of 2 x %d values that layer_norm returned" % rows)
    lib = load_library()
    need = lib.sc_layernorm_workspace_bytes(rows, cols)
    with _Queue(X, stream) as q:
        out = q.empty((rows, cols), X.dtype) if out is None else out
        dweight = q.empty((cols,), torch.float32) if dweight is None else dweight
        dbias = q.empty((cols,), torch.float32) if dbias is None else dbias
        workspace = q.empty((need,), torch.uint8) if workspace is None else workspace
        lddx = _matrix("out", out, (rows, cols), X.dtype, dev)
        ws = _buffer("workspace", workspace, need, dev)
        _check(lib.sc_layernorm_backward(dY.data_ptr(), X.data_ptr(), _DTYPES[X.dtype], w, stats.data_ptr(),
                                         _ptr(residual_grad), out.data_ptr(), _vector("dweight", dweight, cols, dev),
                                         _vector("dbias", dbias, cols, dev), rows, cols, lddy, ldx, ldr, lddx, ws,
                                         workspace.numel(), q.stream.cuda_stream), "sc_layernorm_backward")
    return out, dweight, dbias


def act8_compress(X, out=None, stream=None) -> Act8:
    """X (bf16 or fp32) as an 8-bit checkpoint."""
    ldx = _matrix("X", X)
    tokens, features = X.shape
    with _Queue(X, stream) as q:
        out = Act8(tokens, features, q.empty((Act8.nbytes(tokens, features),), torch.uint8)) if out is None else out
        a8 = _saved("out", out, tokens, features, X.device)
        _check(load_library().sc_act8_compress(X.data_ptr(), _DTYPES[X.dtype], a8, tokens, features, ldx,
                                               q.stream.cuda_stream), "sc_act8_compress")
    return out


def act8_expand(saved, act="none", out=None, out_dtype=torch.bfloat16, stream=None):
    """act(v) of the values v a checkpoint stands for (act "none": the values, exact in bf16)."""
    a = _act(act)
    with _Queue(saved.data, stream) as q:
        out = q.empty((saved.tokens, saved.features), out_dtype) if out is None else out
        ldy = _matrix("out", out, (saved.tokens, saved.features), None, saved.data.device)
        _check(load_library().sc_act8_expand(saved.data.data_ptr(), a, out.data_ptr(), _DTYPES[out.dtype], saved.tokens,
                                             saved.features, ldy, q.stream.cuda_stream), "sc_act8_expand")
    return out


def act8_backward(dA, saved, act, out=None, stream=None):
    """dZ = dA * act'(v): the gradient through an activation whose argument was kept in 8 bits. out may be dA."""
    a = _act(act)
    ldda = _matrix("dA", dA)
    tokens, features = dA.shape
    a8 = _saved("saved", saved, tokens, features, dA.device)
    if a8 is None:
        raise ValueError("saved must be an Act8")
    with _Queue(dA, stream) as q:
        out = q.empty((tokens, features), dA.dtype) if out is None else out
        lddz = _matrix("out", out, (tokens, features), dA.dtype, dA.device)
        _check(load_library().sc_act8_backward(dA.data_ptr(), a8, a, out.data_ptr(), _DTYPES[dA.dtype], tokens, features,
                                               ldda, lddz, q.stream.cuda_stream), "sc_act8_backward")
    return out


def linear(X, W, bias=None, residual=None, act="none", save=None, out=None, out_dtype=None, status=None, stream=None):
    """Y = act(X W^T + bias) + residual in one kernel. X: tokens x cols, W: rows x cols, both bf16 (tensor cores) or both
    fp32. save: an Act8 of tokens x rows that receives X W^T + bias in 8 bits for the backward pass. out_dtype defaults to
    X's; residual has the output's type; out may be residual."""
    a = _act(act)
    ldx = _matrix("X", X)
    dev = X.device
    ldw = _matrix("W", W, None, X.dtype, dev)
    (tokens, cols), rows = X.shape, W.shape[0]
    if W.shape[1] != cols:
        raise ValueError("W has shape %s, expected (rows, %d)" % (tuple(W.shape), cols))
    out_dtype = out.dtype if out is not None else X.dtype if out_dtype is None else out_dtype
    ldr = _matrix("residual", residual, (tokens, rows), out_dtype, dev) if residual is not None else 0
    b = _vector("bias", bias, rows, dev)
    a8 = _saved("save", save, tokens, rows, dev)
    with _Queue(X, stream) as q:
        out = q.empty((tokens, rows), out_dtype) if out is None else out
        ldy = _matrix("out", out, (tokens, rows), None, dev)
        _check(load_library().sc_linear_forward(X.data_ptr(), W.data_ptr(), _DTYPES[X.dtype], b, _ptr(residual),
                                                out.data_ptr(), _DTYPES[out_dtype], a, a8, tokens, rows, cols, ldx, ldw,
                                                ldr, ldy, _status(status, dev), q.stream.cuda_stream), "sc_linear_forward")
    return out


def linear_backward_input(dY, W, saved=None, act="none", out=None, out_dtype=None, status=None, stream=None):
    """dX = dY W; with `saved` (an Act8 of tokens x cols: the pre-activation this layer's input came from)
    dX = (dY W) * act'(v), that pre-activation's gradient, in one kernel."""
    a = _act(act)
    lddy = _matrix("dY", dY)
    dev = dY.device
    ldw = _matrix("W", W, None, dY.dtype, dev)
    (tokens, rows), cols = dY.shape, W.shape[1]
    if W.shape[0] != rows:
        raise ValueError("W has shape %s, expected (%d, cols)" % (tuple(W.shape), rows))
    out_dtype = out.dtype if out is not None else dY.dtype if out_dtype is None else out_dtype
    a8 = _saved("saved", saved, tokens, cols, dev)
    with _Queue(dY, stream) as q:
        out = q.empty((tokens, cols), out_dtype) if out is None else out
        lddx = _matrix("out", out, (tokens, cols), None, dev)
        _check(load_library().sc_linear_backward_input(dY.data_ptr(), W.data_ptr(), _DTYPES[dY.dtype], a8, a,
                                                       out.data_ptr(), _DTYPES[out_dtype], tokens, rows, cols, lddy, ldw,
                                                       lddx, _status(status, dev), q.stream.cuda_stream),
               "sc_linear_backward_input")
    return out


def linear_weight_grad(dY, saved, act="none", scale: float = 1.0, out=None, out_dtype=None, dbias=None, workspace=None,
                       status=None, stream=None):
    """(G, dbias): G = scale * dY^T act(v) (rows x cols, dY's type unless out / out_dtype say otherwise) and the sum of dY
    over the tokens (fp32, not scaled), from the layer's input or pre-activation kept in 8 bits. workspace: uint8,
    sc_linear_weight_grad_workspace_bytes(dtype, tokens, rows, cols)."""
    a = _act(act)
    lddy = _matrix("dY", dY)
    dev = dY.device
    tokens, rows = dY.shape
    if not isinstance(saved, Act8):
        raise ValueError("saved must be an Act8")
    cols = saved.features
    a8 = _saved("saved", saved, tokens, cols, dev)
    out_dtype = out.dtype if out is not None else dY.dtype if out_dtype is None else out_dtype
    lib = load_library()
    dt = _DTYPES[dY.dtype]
    need = lib.sc_linear_weight_grad_workspace_bytes(dt, tokens, rows, cols)
    if need == 0:
        raise SCError(-2, "sc_linear_weight_grad_workspace_bytes")
    with _Queue(dY, stream) as q:
        out = q.empty((rows, cols), out_dtype) if out is None else out
        if _matrix("out", out, (rows, cols), None, dev) != cols:
            raise ValueError("out must be contiguous")
        dbias = q.empty((rows,), torch.float32) if dbias is None else dbias
        workspace = q.empty((need,), torch.uint8) if workspace is None else workspace
        ws = _buffer("workspace", workspace, need, dev)
        _check(lib.sc_linear_weight_grad(dY.data_ptr(), dt, a8, a, float(scale), out.data_ptr(), _DTYPES[out_dtype],
                                         _vector("dbias", dbias, rows, dev), tokens, rows, cols, lddy, ws,
                                         workspace.numel(), _status(status, dev), q.stream.cuda_stream),
               "sc_linear_weight_grad")
    return out, dbias
