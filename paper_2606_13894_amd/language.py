"""A language model's two ends on the library's kernels: tokens to rows, dropout, and log
probabilities over the vocabulary.

* :func:`embedding` / :func:`embedding_backward` -- rows of a table, and the table's gradient.
* :func:`dropout` -- a mask that is a function of a seed and the element's index, never stored;
  the same call on the gradient is its backward pass.
* :func:`token_logprobs` / :func:`token_logprobs_backward` -- from rows of scores, the log
  probabilities of given tokens, the entropy and the best alternatives.
* :func:`head_logprobs` / :func:`head_logprobs_backward` -- the first two from hidden states and
  the output head's weight, the scores never stored.
* :class:`Embedding`, :class:`Dropout`, :class:`LogProbs`, :class:`Head` -- the same under
  autograd.

``include/gefen.h`` gives each operator's formula, types and limits. Tokens are int32 or int64
device tensors; one below 0 stands for none (padding, a position without a loss), one from the
vocabulary's size on makes NaN of what it asks for. As in ``feed_forward.py`` tensors may have any
leading dimensions, calls are asynchronous on ``stream`` (the current torch stream by default), and
where an argument of a plain call wants a gradient, a gradient through its results is an error.

Calls and modules can be captured into graphs, backward passes too (``torch.autograd.grad``, or
``backward`` after a warm-up on a side stream). As with any module, no eager result that still holds
its autograd graph over the same parameters may be kept while a backward pass is captured.
"""
from __future__ import annotations

import ctypes
import operator
from typing import NamedTuple, Optional

import torch

from . import feed_forward as ff

_TOKEN_BYTES = {torch.int32: 4, torch.int64: 8}
_NO_GRADIENT = "{} has no gradient of its own: {} has (or call it under torch.no_grad())"


def _tokens(t, dev, shape=None):
    """tokens, contiguous, and their size in bytes, after their checks."""
    size = _TOKEN_BYTES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if isinstance(t, torch.Tensor) and size is None:
        raise TypeError(f"tokens must be int32 or int64, not {t.dtype}")
    return ff._operand(t, "tokens", dev, None, shape), size


def _table_size(vocab, width):
    if vocab < 1 or width < 1:
        raise ValueError("a table has at least one row of at least one element")


def _space(query, like, *sizes):
    """The workspace that `query` asks for, its address and its size."""
    n = ctypes.c_int64()
    ff._call(query(*sizes, n))
    n = n.value
    if not n:
        return None, None, 0
    ws = like.new_empty(n, dtype=torch.uint8)
    return ws, ws.data_ptr(), n


def _row_results(tokens):
    """Three float32 outputs, one number per token each."""
    a = torch.empty_like(tokens, dtype=torch.float32)
    return a, torch.empty_like(a), torch.empty_like(a)


# ------------------------------------------------------------------ embedding
def embedding(tokens, table, scale: float = 1.0, dtype=None, stream=None):
    """scale * table[tokens] (zeros where a token is below 0), of shape (*tokens.shape, width), in
    ``dtype``: float32 or bfloat16, the table's by default."""
    if stream is not None:
        return ff._on(stream, embedding, tokens, table, scale, dtype)
    dev = ff._device(tokens, "tokens")
    tokens, size = _tokens(tokens, dev)
    table = ff._operand(table, "table", dev)
    if table.dim() != 2:
        raise ValueError(f"table has shape {tuple(table.shape)}, expected (vocab, width)")
    vocab, width = table.shape
    _table_size(vocab, width)
    td = ff._dtype(table, "table")
    y = table.new_empty((*tokens.shape, width), dtype=dtype or table.dtype)
    ff._call(ff._library().gefen_embedding(
        tokens.data_ptr(), size, tokens.numel(), table.data_ptr(), td, vocab, width, scale,
        y.data_ptr(), ff._dtype(y, "y"), ff._raw_stream(dev)))
    if ff._tracked(table):
        ff._no_graph(_NO_GRADIENT.format("embedding", "Embedding"), y)
    return y


def embedding_backward(dy, tokens, vocab: int, scale: float = 1.0, dtype=torch.float32,
                       stream=None):
    """The gradient of :func:`embedding`'s table: (vocab, width) of ``dtype``, each row the sum
    in float32 of scale * dy over its tokens, in an order that the tokens alone decide."""
    if stream is not None:
        return ff._on(stream, embedding_backward, dy, tokens, vocab, scale, dtype)
    dev = ff._device(dy, "dy")
    dy = ff._operand(dy, "dy", dev)
    d = ff._dtype(dy, "dy")
    if not dy.dim():
        raise ValueError("dy must have rows of at least one element")
    tokens, size = _tokens(tokens, dev, dy.shape[:-1])
    width = dy.shape[-1]
    _table_size(vocab, width)
    out = dy.new_empty((vocab, width), dtype=dtype)
    lib = ff._library()
    ws, wp, n = _space(lib.gefen_embedding_backward_workspace, dy, tokens.numel(), vocab, width)
    ff._call(lib.gefen_embedding_backward(
        dy.data_ptr(), d, tokens.data_ptr(), size, tokens.numel(), vocab, width, scale,
        out.data_ptr(), ff._dtype(out, "dtable"), wp, n, ff._raw_stream(dev)))
    if ff._tracked(dy):
        ff._no_graph(ff._BACKWARD_ONLY.format("embedding_backward"), out)
    return out


class _Lookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, scale, dtype):
        ctx.save_for_backward(tokens)
        ctx.table, ctx.scale = (table.shape[0], table.dtype), scale
        return embedding(tokens, table, scale, dtype)

    @staticmethod
    def backward(ctx, dy):
        with torch.no_grad():
            vocab, dtype = ctx.table
            g = embedding_backward(dy, ctx.saved_tensors[0], vocab, ctx.scale, dtype)
        if torch.is_grad_enabled():   # create_graph
            ff._no_graph("Embedding has no second derivative", g)
        return g, None, None, None


class Embedding(torch.nn.Module):
    """``rows = emb(tokens)``: bfloat16 rows of the float32 parameter ``table``, times ``scale``."""

    def __init__(self, vocab: int, width: int, scale: float = 1.0, device=None):
        super().__init__()
        self.scale = scale
        self.table = torch.nn.Parameter(torch.randn(vocab, width, device=device) * 0.02)

    def forward(self, tokens):
        return _Lookup.apply(self.table, tokens, self.scale, torch.bfloat16)


# ------------------------------------------------------------------ dropout
def dropout(x, p: float, seed, offset: int = 0, residual=None, stream=None):
    """x with a share p of its elements (in steps of 2^-16) set to zero and the others scaled to
    keep the mean, plus ``residual``. Which ones depends on ``seed``, ``offset`` and an element's index
    alone, so that the gradient of x is ``dropout(dy, p, seed, offset)``; other calls take other
    offsets. ``seed`` is a number, or an int64 device tensor (seed, a number added to offset) that
    is read when the kernel runs."""
    if stream is not None:
        return ff._on(stream, dropout, x, p, seed, offset, residual)
    dev = ff._device(x, "x")
    x = ff._operand(x, "x", dev)
    d = ff._dtype(x, "x")
    rp = sp = None
    number = 0
    if isinstance(seed, torch.Tensor):
        seed = ff._operand(seed, "seed", dev, torch.int64, (2,))
        sp = seed.data_ptr()
    else:
        number = operator.index(seed) & 0xFFFFFFFFFFFFFFFF
    if residual is not None:
        residual = ff._operand(residual, "residual", dev, x.dtype, x.shape)
        rp = residual.data_ptr()
    y = torch.empty_like(x)
    ff._call(ff._library().gefen_dropout(
        x.data_ptr(), rp, d, x.numel(), p, number, operator.index(offset) & 0xFFFFFFFFFFFFFFFF, sp,
        y.data_ptr(), ff._raw_stream(dev)))
    if ff._tracked(x, residual):
        ff._no_graph(_NO_GRADIENT.format("dropout", "Dropout"), y)
    return y


class _Drop(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, state):
        ctx.save_for_backward(state)
        ctx.p, ctx.residual = p, residual is not None
        return dropout(x, p, state, residual=residual)

    @staticmethod
    def backward(ctx, dy):
        dx = None
        if ctx.needs_input_grad[0]:
            with torch.no_grad():
                dx = dropout(dy, ctx.p, ctx.saved_tensors[0])
            if torch.is_grad_enabled():   # create_graph
                ff._no_graph("Dropout has no second derivative", dx)
        return dx, dy if ctx.residual else None, None, None


class Dropout(torch.nn.Module):
    """``y = drop(x, residual)`` in training: :func:`dropout` with the next offset each time. The
    buffer ``state`` (seed, next offset) lies on the device, so that a captured training step
    drops other elements in each replay, and a saved state resumes. Without ``seed`` the first training
    pass draws one from torch's host generator where the state is new (two zeros), so that the modules of a
    model drop different elements, and the same ones in each run after ``torch.manual_seed``; copies
    of a module that has run drop what it drops. Evaluation, and p = 0, give x (plus residual). A
    training pass that is run again within a backward pass, in the place of saved activations
    (``torch.utils.checkpoint``), is an error: it would take the next offset, and drop other elements
    than the first time. (Where a wrapper makes the buffers of all ranks those of rank 0, all of them drop
    the same elements.)"""

    _draw = False       # whether the next training pass draws the seed

    def __init__(self, p: float = 0.1, seed: Optional[int] = None, device=None):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must be in [0, 1]")
        self.p = p
        self._draw = self._draws = seed is None
        self.register_buffer("state", torch.tensor([seed or 0, 0], dtype=torch.int64,
                                                   device=device))

    def _load_from_state_dict(self, *args):
        super()._load_from_state_dict(*args)
        self._draw = self.__dict__.get("_draws", False)

    def _draw_seed(self):
        # decided on the device: a state that was loaded, or has moved on between replays, stays
        seed = torch.randint(1, 2 ** 63 - 1, (), device="cpu").item()
        self.state[:1].masked_fill_((self.state[:1] == 0) & (self.state[1:] == 0), seed)
        # (what was captured has not run yet)
        self._draw = self.state.device.type == "cuda" and torch.cuda.is_current_stream_capturing()

    def forward(self, x, residual=None):
        if not self.training or self.p == 0.0:
            return x if residual is None else x + residual
        if torch._C._current_graph_task_id() != -1:
            raise RuntimeError("Dropout is run again within a backward pass: it would drop other "
                               "elements than the first time (leave it out of what is recomputed)")
        if self._draw:
            self._draw_seed()
        state = self.state.clone()
        self.state[1:].add_(1)
        return _Drop.apply(x, residual, self.p, state)


# ------------------------------------------------------------------ log probabilities
class TokenLogProbs(NamedTuple):
    """float32, one per row: ``logprob`` of the row's token, ``entropy``, ``lse`` the log of the
    sum of exponentials; with alternatives ``top_logprobs`` and ``top_tokens`` (int64), from the
    largest down."""
    logprob: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logprobs: Optional[torch.Tensor]
    top_tokens: Optional[torch.Tensor]


def _score_rows(z, what, dev):
    """z as rows x vocab whose rows lie evenly apart, a copy only where they do not."""
    if not isinstance(z, torch.Tensor) or not z.is_cuda or z.get_device() != dev:
        ff._operand(z, what, dev)
    if not z.dim() or not z.shape[-1]:
        raise ValueError(f"{what} must have rows of at least one element")
    if z.dim() == 2 and z.is_contiguous():
        return z, z.shape[1]
    rows = z.reshape(-1, z.shape[-1]) if z.numel() else z.new_empty((0, z.shape[-1]))
    if rows.shape[0] == 1 and rows.stride(1) == 1:
        return rows, rows.shape[1]
    if rows.stride(1) != 1 or rows.stride(0) < rows.shape[1]:
        rows = rows.contiguous()
    return rows, rows.stride(0)


def token_logprobs(logits, tokens, top: int = 0, stream=None):
    """:class:`TokenLogProbs` of float32 or bfloat16 rows of scores (..., vocab) and one token
    for each, with the ``top`` (at most 32) best alternatives, equal ones from the lowest token
    up. A mask is -inf in the scores. Rows may lie further apart than they are long
    (``padded[..., :vocab]``)."""
    if stream is not None:
        return ff._on(stream, token_logprobs, logits, tokens, top)
    return _token_logprobs(logits, tokens, top, False)[0]


def _token_logprobs(logits, tokens, top, split):
    """The results, and with ``split`` what rounding left of lse."""
    dev = ff._device(logits, "logits")
    d = ff._dtype(logits, "logits")
    z, ld = _score_rows(logits, "logits", dev)
    rows, vocab = z.shape
    shape = logits.shape[:-1]
    tokens, size = _tokens(tokens, dev, shape)
    if not 0 <= top <= min(32, vocab):
        raise ValueError(f"top must be in [0, {min(32, vocab)}]")
    logprob, entropy, lse = _row_results(tokens)
    best = where = bp = kp = None
    if top:
        best = lse.new_empty((*shape, top))
        where = tokens.new_empty((*shape, top), dtype=torch.int64)
        bp, kp = best.data_ptr(), where.data_ptr()
    lib = ff._library()
    ws, wp, n = _space(lib.gefen_token_logprobs_workspace, z, d, rows, vocab, top)
    rest = torch.empty_like(lse) if split else None
    entry, more = (lib.gefen_token_logprobs_split, (rest.data_ptr(),)) if split else (
        lib.gefen_token_logprobs, ())
    ff._call(entry(
        z.data_ptr(), ld, d, rows, vocab, tokens.data_ptr(), size, top, logprob.data_ptr(),
        entropy.data_ptr(), lse.data_ptr(), *more, bp, kp, wp, n, ff._raw_stream(dev)))
    if ff._tracked(logits):
        ff._no_graph(_NO_GRADIENT.format("token_logprobs", "LogProbs"), logprob, entropy, lse,
                     *((best,) if top else ()))
    return TokenLogProbs(logprob, entropy, lse, best, where), rest


def _upstream(dlogprob, dentropy, dev, shape):
    """The gradients' addresses and what keeps them alive."""
    f32 = torch.float32
    g = ff._operand(dlogprob, "dlogprob", dev, f32, shape)
    h = None if dentropy is None else ff._operand(dentropy, "dentropy", dev, f32, shape)
    return g, h, g.data_ptr(), None if h is None else h.data_ptr()


def token_logprobs_backward(dlogprob, logits, tokens, lse, entropy, dentropy=None, out=None,
                            stream=None):
    """The gradient of :func:`token_logprobs`'s logits from those of logprob and entropy. ``out``
    takes it (contiguous, or rows evenly apart, no gradient wanted of it); it may be ``logits``
    itself. The probabilities are exp(logits - lse), off by |lse| 2^-24 of them, since lse is rounded: rows
    far from 0, as a finite mask over all of one leaves it, are for :class:`LogProbs`, which keeps what
    rounding left of lse."""
    if stream is not None:
        return ff._on(stream, token_logprobs_backward, dlogprob, logits, tokens, lse, entropy,
                      dentropy, out)
    return _token_logprobs_backward(dlogprob, logits, tokens, lse, None, entropy, dentropy, out)


def _token_logprobs_backward(dlogprob, logits, tokens, lse, rest, entropy, dentropy, out):
    dev = ff._device(logits, "logits")
    d = ff._dtype(logits, "logits")
    z, ld = _score_rows(logits, "logits", dev)
    rows, vocab = z.shape
    shape = logits.shape[:-1]
    tokens, size = _tokens(tokens, dev, shape)
    f32 = torch.float32
    lse = ff._operand(lse, "lse", dev, f32, shape)
    entropy = ff._operand(entropy, "entropy", dev, f32, shape)
    g, h, gp, hp = _upstream(dlogprob, dentropy, dev, shape)
    if out is None:
        out = torch.empty_like(z) if z is logits else logits.new_empty(logits.shape)
        to, ldd = out, vocab
    else:
        if not isinstance(out, torch.Tensor) or out.dtype is not logits.dtype or \
                out.shape != logits.shape:
            raise ValueError(f"out must be {logits.dtype} of shape {tuple(logits.shape)}")
        if out.requires_grad:
            raise ValueError("out is written in place and must not want a gradient")
        to, ldd = _score_rows(out, "out", dev)
        if to.data_ptr() != out.data_ptr():
            raise ValueError("out must have its rows evenly apart")
        torch.autograd.graph.increment_version(out)   # what was saved of it is gone
    lib = ff._library()
    entry, more = (lib.gefen_token_logprobs_backward, ()) if rest is None else (
        lib.gefen_token_logprobs_backward_split, (rest.data_ptr(),))
    ff._call(entry(
        z.data_ptr(), ld, d, rows, vocab, tokens.data_ptr(), size, lse.data_ptr(), *more,
        entropy.data_ptr(), gp, hp, to.data_ptr(), ldd, ff._raw_stream(dev)))
    if ff._tracked(dlogprob, dentropy, logits):
        ff._no_graph(ff._BACKWARD_ONLY.format("token_logprobs_backward"), out)
    return out


def _of_logprob(g, like):
    """The log probabilities' gradient, zeros where none of them was used."""
    return torch.zeros_like(like) if g is None else g


class _Scores(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens):
        r, rest = _token_logprobs(logits, tokens, 0, True)
        ctx.save_for_backward(logits, tokens, r.lse, rest, r.entropy)
        ctx.set_materialize_grads(False)
        return r.logprob, r.entropy

    @staticmethod
    def backward(ctx, dlogprob, dentropy):
        logits, tokens, lse, rest, entropy = ctx.saved_tensors
        with torch.no_grad():
            dz = _token_logprobs_backward(_of_logprob(dlogprob, lse), logits, tokens, lse, rest,
                                          entropy, dentropy, None)
        if torch.is_grad_enabled():   # create_graph
            ff._no_graph("LogProbs has no second derivative", dz)
        return dz, None


class LogProbs(torch.nn.Module):
    """``logprob, entropy = scores(logits, tokens)`` of :func:`token_logprobs`, under autograd."""

    def forward(self, logits, tokens):
        return _Scores.apply(logits, tokens)


# ------------------------------------------------------------------ output head
class HeadLogProbs(NamedTuple):
    """float32, one per row: ``logprob`` of the row's token, ``entropy``, ``lse``."""
    logprob: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor


def _head_operands(x, weight, tokens):
    dev = ff._device(x, "x")
    bf16 = torch.bfloat16
    x = ff._operand(x, "x", dev, bf16)
    n, width = ff._rows(x, "x")
    weight = ff._operand(weight, "weight", dev, bf16)
    if weight.dim() != 2 or weight.shape[1] != width or weight.shape[0] < 1:
        raise ValueError(f"weight has shape {tuple(weight.shape)}, expected (vocab, {width})")
    tokens, size = _tokens(tokens, dev, x.shape[:-1])
    return dev, x, weight, tokens, size, n, width, weight.shape[0]


def _head_space(lib, x, weight, n, width, vocab, flags):
    if (x.data_ptr() | weight.data_ptr()) & 15:
        flags |= ff._UNALIGNED
    return _space(lib.gefen_head_logprobs_workspace, x, n, width, vocab, flags)


def head_logprobs(x, weight, tokens, stream=None):
    """:class:`HeadLogProbs` of the scores x weight^T, which are never stored: x bfloat16 hidden
    states (..., width), weight bfloat16 (vocab, width), one token for each row."""
    if stream is not None:
        return ff._on(stream, head_logprobs, x, weight, tokens)
    wants = ff._tracked(x, weight)
    dev, x, weight, tokens, size, n, width, vocab = _head_operands(x, weight, tokens)
    lib = ff._library()
    logprob, entropy, lse = _row_results(tokens)
    ws, wp, nb = _head_space(lib, x, weight, n, width, vocab, 0)
    ff._call(lib.gefen_head_logprobs(
        x.data_ptr(), weight.data_ptr(), tokens.data_ptr(), size, n, width, vocab,
        logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), wp, nb, ff._raw_stream(dev)))
    if wants:
        ff._no_graph(_NO_GRADIENT.format("head_logprobs", "Head"), logprob, entropy, lse)
    return HeadLogProbs(logprob, entropy, lse)


def head_logprobs_backward(dlogprob, x, weight, tokens, lse, entropy, dentropy=None,
                           x_grad: bool = True, weight_grad: bool = True, stream=None):
    """(dx, dweight) of :func:`head_logprobs`, bfloat16, from the gradients of logprob and entropy;
    None in the place of one that is not asked for. The scores are formed again, for a range of the
    vocabulary at a time."""
    if stream is not None:
        return ff._on(stream, head_logprobs_backward, dlogprob, x, weight, tokens, lse, entropy,
                      dentropy, x_grad, weight_grad)
    if not x_grad and not weight_grad:
        raise ValueError("neither gradient is asked for")
    wants = ff._tracked(dlogprob, dentropy, x, weight)
    dev, x, weight, tokens, size, n, width, vocab = _head_operands(x, weight, tokens)
    shape = x.shape[:-1]
    lse = ff._operand(lse, "lse", dev, torch.float32, shape)
    entropy = ff._operand(entropy, "entropy", dev, torch.float32, shape)
    g, h, gp, hp = _upstream(dlogprob, dentropy, dev, shape)
    lib = ff._library()
    dx = torch.empty_like(x) if x_grad else None
    dw = torch.empty_like(weight) if weight_grad else None
    ws, wp, nb = _head_space(lib, x, weight, n, width, vocab, ff._BACKWARD)
    ff._call(lib.gefen_head_logprobs_backward(
        x.data_ptr(), weight.data_ptr(), tokens.data_ptr(), size, n, width, vocab, lse.data_ptr(),
        entropy.data_ptr(), gp, hp, dx.data_ptr() if x_grad else None,
        dw.data_ptr() if weight_grad else None, wp, nb, ff._raw_stream(dev)))
    if wants:
        ff._no_graph(ff._BACKWARD_ONLY.format("head_logprobs_backward"),
                     *(g for g in (dx, dw) if g is not None))
    return dx, dw


class _HeadScores(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, tokens):
        r = head_logprobs(x, weight, tokens)
        ctx.save_for_backward(x, weight, tokens, r.lse, r.entropy)
        ctx.set_materialize_grads(False)
        return r.logprob, r.entropy

    @staticmethod
    def backward(ctx, dlogprob, dentropy):
        x, weight, tokens, lse, entropy = ctx.saved_tensors
        with torch.no_grad():
            dx, dw = head_logprobs_backward(_of_logprob(dlogprob, lse), x, weight, tokens, lse,
                                            entropy, dentropy, *ctx.needs_input_grad[:2])
        if torch.is_grad_enabled():   # create_graph
            ff._no_graph("Head has no second derivative",
                         *(g for g in (dx, dw) if g is not None))
        return dx, dw, None


class Head(torch.nn.Module):
    """``logprob, entropy = head(x, tokens)``: the log probabilities of the tokens that follow and
    the entropies, over the float32 parameter ``weight`` (vocab, width), which each call casts to
    bfloat16 and may be another module's (``Head(..., weight=emb.table)``: its gradient is then the
    sum). The mean of -logprob over the tokens that count is the usual loss. (The cast and the gradient's
    back take 0.27 ms each at 128256 x 2048, of 13.1 ms for 8192 tokens. A program that serves casts the weight
    once and calls :func:`head_logprobs` itself.)"""

    def __init__(self, width: int, vocab: int, weight=None, device=None):
        super().__init__()
        if weight is None:
            weight = torch.nn.Parameter(torch.randn(vocab, width, device=device) * width ** -0.5)
        elif weight.shape != (vocab, width):
            raise ValueError(f"weight has shape {tuple(weight.shape)}, expected {(vocab, width)}")
        self.weight = weight

    def forward(self, x, tokens):
        return _HeadScores.apply(x, self.weight.to(torch.bfloat16), tokens)
