"""The feed-forward half of a transformer block on the library's kernels, trained with one byte
per saved activation.

* :func:`checkpoint8` / :meth:`Checkpoint8.decode` -- 8-bit activation checkpoints.
* :func:`rms_norm` / :func:`rms_norm_backward` -- the residual's addition and RMS norm, with an
  8-bit checkpoint of the normalised rows.
* :func:`gated_ffn` / :func:`gated_ffn_backward` -- the gated block, with 8-bit checkpoints of
  its gate and up activations.
* :class:`FeedForward` -- all of it as one module under autograd.

``include/gefen.h`` gives each operator's formula, types and limits. Tensors are device tensors
of any leading dimensions (rows are all but the last); ones that are not contiguous are copied.
All calls are asynchronous on ``stream`` (the current torch stream by default), where their
outputs and workspaces are allocated. Only ``FeedForward`` has an autograd form: where an
argument of the other calls wants a gradient, a gradient through their results is an error.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import BF16, F32, _check, load_library

GROUP = 64
ACTIVATIONS = {"silu": 0, "gelu": 1}
_BACKWARD, _UNALIGNED = 1, 2

_DTYPE = {torch.float32: F32, torch.bfloat16: BF16}


_raw_stream = torch._C._cuda_getCurrentRawStream   # no Stream object: a microsecond less a call
_current_device = torch._C._cuda_getDevice         # for callers that hold a device tensor already
_lib = None


def _library():
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


def _on(stream, fn, *args):
    """fn(*args) with `stream` as torch's current stream."""
    with torch.cuda.stream(stream):
        return fn(*args)


def _device(t, what):
    """The index of t's device, which is the current one."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    dev = t.get_device()
    if dev != _current_device():
        raise ValueError(f"{what} is on {t.device}, not on the current device")
    return dev


def _operand(t, what, dev, dtype=None, shape=None):
    """t, contiguous, after its checks."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.get_device() != dev:
        raise ValueError(f"{what} is on {t.device}, not on the current device")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{what} must be {dtype}, not {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t if t.is_contiguous() else t.contiguous()


def _rows(t, what):
    """(rows, cols) of a tensor whose last dimension is a row."""
    shape = t.shape
    if len(shape) == 2 and shape[1]:
        return shape
    if not shape or not shape[-1]:
        raise ValueError(f"{what} must have rows of at least one element")
    return t.numel() // shape[-1], shape[-1]


def _dtype(t, what):
    d = _DTYPE.get(t.dtype)
    if d is None:
        raise TypeError(f"{what} must be float32 or bfloat16, not {t.dtype}")
    return d


def _call(code):
    if code:
        _check(code)


def _saved(c, what, dev, shape):
    """The codes' and exponents' addresses of checkpoint c, after its checks."""
    if not isinstance(c, Checkpoint8) or c.codes.shape != shape:
        raise ValueError(f"{what} must be a Checkpoint8 of shape {tuple(shape)}")
    if c.codes.get_device() != dev:
        raise ValueError(f"{what} is on {c.codes.device}, not on the current device")
    return c.codes.data_ptr(), c.exponents.data_ptr()


class _NoGraph(torch.autograd.Function):
    """A kernel's result under autograd: it carries no graph, so that a gradient through it is an
    error and not a missing share. The tensor itself is returned."""

    @staticmethod
    def forward(ctx, anchor, what, result):
        ctx.what = what
        ctx.mark_dirty(result)
        return result

    @staticmethod
    def backward(ctx, grad):
        raise RuntimeError(ctx.what)


def _no_graph(what, *results):
    anchor = torch.ones((), requires_grad=True)
    for r in results:
        _NoGraph.apply(anchor, what, r)


def _tracked(*tensors):
    """Whether autograd would want a graph from them to the results."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


_FORWARD = " has no gradient of its own: FeedForward has (or call it under torch.no_grad())"
_BACKWARD_ONLY = "the results of {} cannot be differentiated"


class Checkpoint8:
    """An 8-bit checkpoint of a tensor: ``codes`` int8, shaped as it, and ``exponents`` uint8, one
    per group of 64 elements of the last dimension. Element = code * 2^(exponent - 127)."""

    __slots__ = ("codes", "exponents")

    def __init__(self, codes, exponents):
        if codes.dtype is not torch.int8 or exponents.dtype is not torch.uint8:
            raise TypeError("codes must be int8 and exponents uint8")
        rows, cols = _rows(codes, "codes")
        if tuple(exponents.shape) != (*codes.shape[:-1], -(-cols // GROUP)):
            raise ValueError(f"exponents have shape {tuple(exponents.shape)}, expected "
                             f"{(*codes.shape[:-1], -(-cols // GROUP))}")
        dev = _device(codes, "codes")
        self.codes = _operand(codes, "codes", dev)
        self.exponents = _operand(exponents, "exponents", dev)

    @classmethod
    def like(cls, t, cols=None):
        """One of t's shape (its last dimension `cols`, if given) and device, to be written."""
        self = cls.__new__(cls)
        shape = t.shape
        if cols is None or cols == shape[-1]:
            cols = shape[-1]
            self.codes = torch.empty_like(t, dtype=torch.int8)
        else:
            self.codes = t.new_empty((*shape[:-1], cols), dtype=torch.int8)
        self.exponents = t.new_empty((*shape[:-1], -(-cols // GROUP)), dtype=torch.uint8)
        return self

    @property
    def shape(self):
        return self.codes.shape

    @property
    def nbytes(self):
        return self.codes.numel() + self.exponents.numel()

    def decode(self, dtype=None, gain=None, out=None, stream=None):
        """The tensor's values (exact in both types), times ``gain`` (float32, one per column), as
        ``dtype``: bfloat16 by default, or ``out``'s, which it is to agree with."""
        if stream is not None:
            return _on(stream, self.decode, dtype, gain, out)
        codes = self.codes
        dev = codes.get_device()
        if dev != _current_device():
            raise ValueError(f"codes are on {codes.device}, not on the current device")
        rows, cols = _rows(codes, "codes")
        if out is None:
            out = torch.empty_like(codes, dtype=dtype or torch.bfloat16)
        elif dtype is not None and out.dtype is not dtype:
            raise TypeError(f"out must be {dtype}, not {out.dtype}")
        elif not out.is_contiguous():
            raise ValueError("out must be contiguous")
        else:
            _operand(out, "out", dev, None, codes.shape)
        d = _dtype(out, "out")
        p = None
        if gain is not None:
            gain = _operand(gain, "gain", dev, torch.float32, (cols,))
            p = gain.data_ptr()
        _call(_library().gefen_checkpoint_decode(codes.data_ptr(), self.exponents.data_ptr(), p,
                                                 rows, cols, out.data_ptr(), d, _raw_stream(dev)))
        if _tracked(gain):
            _no_graph("decode" + _FORWARD, out)
        return out


def checkpoint8(x, stream=None):
    """The 8-bit checkpoint of a float32 or bfloat16 tensor, in groups of 64 along its last
    dimension."""
    if stream is not None:
        return _on(stream, checkpoint8, x)
    dev = _device(x, "x")
    if not x.is_contiguous():
        x = x.contiguous()
    d = _dtype(x, "x")
    rows, cols = _rows(x, "x")
    c = Checkpoint8.like(x)
    _call(_library().gefen_checkpoint_encode(x.data_ptr(), d, rows, cols, c.codes.data_ptr(),
                                             c.exponents.data_ptr(), _raw_stream(dev)))
    return c


class RMSNormOutput(NamedTuple):
    """``y`` the scaled rows; ``h`` = x + residual (x itself without one); ``rstd`` float32, one
    per row; ``checkpoint`` of h * rstd, or None."""
    y: torch.Tensor
    h: torch.Tensor
    rstd: torch.Tensor
    checkpoint: Optional[Checkpoint8]


def rms_norm(x, weight, residual=None, eps: float = 1e-6, checkpoint: bool = False, stream=None):
    """RMS norm of each row of x + residual, times weight (float32): an :class:`RMSNormOutput`.
    With ``checkpoint`` the normalised rows are saved in 8 bits for the backward passes."""
    if stream is not None:
        return _on(stream, rms_norm, x, weight, residual, eps, checkpoint)
    dev = _device(x, "x")
    if not x.is_contiguous():
        x = x.contiguous()
    d = _dtype(x, "x")
    rows, cols = _rows(x, "x")
    weight = _operand(weight, "weight", dev, torch.float32, (cols,))
    y = torch.empty_like(x)
    h, rp, hp = x, None, None
    if residual is not None:
        residual = _operand(residual, "residual", dev, x.dtype, x.shape)
        h = torch.empty_like(x)
        rp, hp = residual.data_ptr(), h.data_ptr()
    rstd = x.new_empty(x.shape[:-1], dtype=torch.float32)
    c = cp = ep = None
    if checkpoint:
        c = Checkpoint8.like(x)
        cp, ep = c.codes.data_ptr(), c.exponents.data_ptr()
    _call(_library().gefen_rms_norm(x.data_ptr(), rp, d, weight.data_ptr(), rows, cols, eps,
                                    y.data_ptr(), hp, rstd.data_ptr(), cp, ep, _raw_stream(dev)))
    if _tracked(x, weight, residual):
        _no_graph("rms_norm" + _FORWARD, y, rstd, *(() if h is x else (h,)))
    return RMSNormOutput(y, h, rstd, c)


def rms_norm_backward(dy, saved, rstd, weight, dh=None, stream=None):
    """(dx, dweight) of :func:`rms_norm`. ``saved`` is its ``checkpoint`` or its ``h``; ``dh`` the
    gradient that h gets from its other uses, added to dx (which is the residual's too)."""
    if stream is not None:
        return _on(stream, rms_norm_backward, dy, saved, rstd, weight, dh)
    dev = _device(dy, "dy")
    if not dy.is_contiguous():
        dy = dy.contiguous()
    d = _dtype(dy, "dy")
    rows, cols = _rows(dy, "dy")
    weight = _operand(weight, "weight", dev, torch.float32, (cols,))
    rstd = _operand(rstd, "rstd", dev, torch.float32, dy.shape[:-1])
    h = codes = exps = None
    if isinstance(saved, Checkpoint8):
        codes, exps = _saved(saved, "saved", dev, dy.shape)
    else:
        saved = _operand(saved, "saved", dev, dy.dtype, dy.shape)
        h = saved.data_ptr()
    p = None
    if dh is not None:
        dh = _operand(dh, "dh", dev, dy.dtype, dy.shape)
        p = dh.data_ptr()
    lib = _library()
    dx = torch.empty_like(dy)
    dw = torch.empty_like(weight)
    n = ctypes.c_int64()
    _call(lib.gefen_rms_norm_backward_workspace(rows, cols, n))
    ws = dy.new_empty(n.value, dtype=torch.uint8)
    _call(lib.gefen_rms_norm_backward(dy.data_ptr(), p, d, h, codes, exps, rstd.data_ptr(),
                                      weight.data_ptr(), rows, cols, dx.data_ptr(), dw.data_ptr(),
                                      ws.data_ptr(), n.value, _raw_stream(dev)))
    if _tracked(dy, dh):
        _no_graph(_BACKWARD_ONLY.format("rms_norm_backward"), dx, dw)
    return dx, dw


def _ffn_operands(rows_of, what, w_gate, w_up, w_down, activation):
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, not {activation!r}")
    dev = _device(rows_of, what)
    bf16 = torch.bfloat16
    t = _operand(rows_of, what, dev, bf16)
    tokens, width = _rows(t, what)
    w_gate = _operand(w_gate, "w_gate", dev, bf16)
    if w_gate.dim() != 2 or w_gate.shape[1] != width or w_gate.shape[0] < 1:
        raise ValueError(f"w_gate has shape {tuple(w_gate.shape)}, expected (inner, {width})")
    inner = w_gate.shape[0]
    w_up = _operand(w_up, "w_up", dev, bf16, (inner, width))
    w_down = _operand(w_down, "w_down", dev, bf16, (width, inner))
    return dev, t, tokens, width, inner, w_gate, w_up, w_down, act


def _ffn_space(lib, like, tokens, width, inner, flags, pointers):
    """The workspace for operands at `pointers`, and its size."""
    for p in pointers:
        if p is not None and p & 15:
            flags |= _UNALIGNED
    n = ctypes.c_int64()
    _call(lib.gefen_gated_ffn_workspace(tokens, width, inner, flags, n))
    return like.new_empty(n.value, dtype=torch.uint8), n.value


def gated_ffn(x, w_gate, w_up, w_down, activation: str = "silu", checkpoint: bool = False,
              stream=None):
    """(act(x w_gate^T) * (x w_up^T)) w_down^T of bfloat16 tensors; weights are [out, in].
    ``activation`` is "silu" or "gelu", the latter in its tanh form (torch's default is the other).
    With ``checkpoint`` returns (y, (gate, up)), the 8-bit checkpoints of both projections for
    :func:`gated_ffn_backward`."""
    if stream is not None:
        return _on(stream, gated_ffn, x, w_gate, w_up, w_down, activation, checkpoint)
    dev, x, tokens, width, inner, w_gate, w_up, w_down, act = _ffn_operands(
        x, "x", w_gate, w_up, w_down, activation)
    lib = _library()
    y = torch.empty_like(x)
    saved, p = None, (None,) * 4
    if checkpoint:
        saved = Checkpoint8.like(x, inner), Checkpoint8.like(x, inner)
        p = tuple(q.data_ptr() for c in saved for q in (c.codes, c.exponents))
    ops = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr()
    ws, n = _ffn_space(lib, x, tokens, width, inner, 0, ops)
    _call(lib.gefen_gated_ffn(*ops, tokens, width, inner, act, y.data_ptr(), *p, ws.data_ptr(), n,
                              _raw_stream(dev)))
    if _tracked(x, w_gate, w_up, w_down):
        _no_graph("gated_ffn" + _FORWARD, y)
    return (y, saved) if checkpoint else y


def gated_ffn_backward(dy, x, saved, w_gate, w_up, w_down, activation: str = "silu", gain=None,
                       stream=None):
    """(dx, dw_gate, dw_up, dw_down) of :func:`gated_ffn` from its checkpoints ``saved``. ``x`` is
    its input, or a :class:`Checkpoint8` of it, times ``gain`` (float32, one per column): the
    checkpoint of the :func:`rms_norm` that made x, with that norm's weight."""
    if stream is not None:
        return _on(stream, gated_ffn_backward, dy, x, saved, w_gate, w_up, w_down, activation,
                   gain)
    dev, dy, tokens, width, inner, w_gate, w_up, w_down, act = _ffn_operands(
        dy, "dy", w_gate, w_up, w_down, activation)
    gate, up = saved
    inside = (*dy.shape[:-1], inner)
    gate = _saved(gate, "the gate's checkpoint", dev, inside)
    up = _saved(up, "the up projection's checkpoint", dev, inside)
    xp = codes = exps = gp = None
    if isinstance(x, Checkpoint8):
        codes, exps = _saved(x, "x", dev, dy.shape)
        if gain is not None:
            gain = _operand(gain, "gain", dev, torch.float32, (width,))
            gp = gain.data_ptr()
    else:
        if gain is not None:
            raise ValueError("gain goes with a Checkpoint8 of x")
        x = _operand(x, "x", dev, torch.bfloat16, dy.shape)
        xp = x.data_ptr()
    lib = _library()
    dx = torch.empty_like(dy)
    dwg, dwu, dwd = (torch.empty_like(w) for w in (w_gate, w_up, w_down))
    dp, w = dy.data_ptr(), (w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr())
    ws, n = _ffn_space(lib, dy, tokens, width, inner, _BACKWARD, (dp, xp, *w))
    _call(lib.gefen_gated_ffn_backward(
        dp, xp, codes, exps, gp, *gate, *up, *w, tokens, width, inner, act, dx.data_ptr(),
        dwg.data_ptr(), dwu.data_ptr(), dwd.data_ptr(), ws.data_ptr(), n, _raw_stream(dev)))
    if _tracked(dy):
        _no_graph(_BACKWARD_ONLY.format("gated_ffn_backward"), dx, dwg, dwu, dwd)
    return dx, dwg, dwu, dwd


class _Block(torch.autograd.Function):
    """y, h = the gated block of rms_norm(x + residual), and h, saved in 8 bits."""

    @staticmethod
    def forward(ctx, x, residual, norm_weight, w_gate, w_up, w_down, eps, activation):
        n = rms_norm(x, norm_weight, residual, eps, checkpoint=True)
        y, (gate, up) = gated_ffn(n.y, w_gate, w_up, w_down, activation, checkpoint=True)
        ctx.save_for_backward(norm_weight, w_gate, w_up, w_down, n.rstd,
                              n.checkpoint.codes, n.checkpoint.exponents, gate.codes,
                              gate.exponents, up.codes, up.exponents)
        ctx.activation, ctx.residual = activation, residual is not None
        return y, (n.h if residual is not None else x.view_as(x))

    @staticmethod
    def backward(ctx, dy, dh):
        nw, wg, wu, wd, rstd, nc, ne, gc, ge, uc, ue = ctx.saved_tensors
        with torch.no_grad():
            saved = Checkpoint8(nc, ne)
            dn, dwg, dwu, dwd = gated_ffn_backward(
                dy, saved, (Checkpoint8(gc, ge), Checkpoint8(uc, ue)), wg, wu, wd,
                ctx.activation, gain=nw)
            dx, dnw = rms_norm_backward(dn, saved, rstd, nw, dh)
        if torch.is_grad_enabled():   # create_graph
            _no_graph("FeedForward has no second derivative", dx, dnw, dwg, dwu, dwd)
        return dx, dx if ctx.residual else None, dnw, dwg, dwu, dwd, None, None


class FeedForward(torch.nn.Module):
    """The feed-forward half of a transformer block: ``y, h = ff(x, residual)`` with
    h = x + residual and y the gated block of the RMS norm of h (so that h + y, or h as the next
    residual of y, goes on). Parameters are float32, as the optimizers take them, and cast to
    bfloat16 in each call; x and residual are bfloat16. A second derivative is an error.

    Kept for the backward pass: the normalised rows and both projections in 8 bits, a float per
    row, and the call's bfloat16 copies of the three weights (6 width inner bytes, more than the
    activations below about 6 width inner / (width + 2 inner) tokens; the casts take 53 us at 2048
    and 8192, and are not done again in the backward pass). Where no gradient is wanted nothing is kept, and
    few tokens take the kernels for them. A program that serves casts the weights once and calls
    :func:`rms_norm` and :func:`gated_ffn` itself.

    ``dropout``: in training y goes through a :class:`Dropout` of that p and ``seed``, whose mask is not
    kept either (a pass over y forward, and one over its gradient), and which cannot be recomputed within
    a backward pass (``torch.utils.checkpoint``): that is an error."""

    def __init__(self, width: int, inner: int, activation: str = "silu", eps: float = 1e-6,
                 device=None, dropout: float = 0.0, seed: Optional[int] = None):
        super().__init__()
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
        self.activation, self.eps = activation, eps
        self.norm = torch.nn.Parameter(torch.ones(width, device=device))

        def weight(out, into):
            return torch.nn.Parameter(torch.randn(out, into, device=device) * into ** -0.5)

        self.w_gate, self.w_up = weight(inner, width), weight(inner, width)
        self.w_down = weight(width, inner)
        self.drop = None
        if dropout:
            from .language import Dropout   # which imports this module
            self.drop = Dropout(dropout, seed, device)

    def __setstate__(self, state):
        super().__setstate__(state)
        if "drop" not in self._modules:     # a module that was pickled before it could have one
            self.__dict__.setdefault("drop", None)

    def forward(self, x, residual=None):
        bf16 = torch.bfloat16
        weights = self.w_gate.to(bf16), self.w_up.to(bf16), self.w_down.to(bf16)
        if _tracked(x, residual, self.norm, *weights):
            y, h = _Block.apply(x, residual, self.norm, *weights, self.eps, self.activation)
        else:
            n = rms_norm(x, self.norm, residual, self.eps)
            y = gated_ffn(n.y, *weights, self.activation)
            h = n.h if residual is not None else x.view_as(x)
        return (y if self.drop is None else self.drop(y)), h
