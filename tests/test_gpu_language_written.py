"""What the entry points write: every element of their outputs whatever was there and in the workspace,
and nothing beside them. Outputs and workspaces are filled with ones (NaN) and lie between guards."""
import ctypes

import pytest
import torch

from test_gpu_language import (BF16, DTYPES, F32, HALF, UNIT, _randint, _randn,  # noqa: F401
                               _table_gradient, _within, dev)

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")

CODE = {F32: 0, BF16: 1}
GUARD = 4096


class Filled:
    """A tensor of ones in all its bits, in the middle of a buffer of the same."""

    def __init__(self, dev, shape, dtype, off=0):
        count = 1
        for n in shape:
            count *= n
        size = torch.empty((), dtype=dtype).element_size()
        self.bytes = torch.full((2 * GUARD + off * size + count * size,), 255, dtype=torch.uint8,
                                device=dev)
        self.at = GUARD + off * size
        self.t = self.bytes[self.at:self.at + count * size].view(dtype).view(shape)
        self.p = self.t.data_ptr() if count else None

    def check(self):
        end = self.at + self.t.numel() * self.t.element_size()
        assert (self.bytes[:self.at] == 255).all() and (self.bytes[end:] == 255).all()
        return self.t


def _call(dev, lib, entry, space, *arguments):
    """The entry with a filled workspace of the size that `space` asks for."""
    n = ctypes.c_int64()
    assert space(n) == 0
    ws = Filled(dev, (n.value,), torch.uint8)
    rc = entry(*arguments, ws.p, n.value, torch.cuda.current_stream(dev).cuda_stream)
    assert rc == 0, lib.gefen_last_error()
    torch.cuda.synchronize()
    ws.check()


@pytest.mark.parametrize("dtype,off", [("bf16", 0), ("f32", 0), ("bf16", 1)])
@pytest.mark.parametrize("n,vocab,width", [
    (0, 50_000, 1001), (0, 3, 1), (1, 1, 1), (5, 50_000, 1001), (1024, 160_001, 517), (1025, 1000, 65),
    (2000, 160_001, 1037), (21_000, 200_000, 1201), (21_000, 300, 40), (70_000, 5000, 9)])
def test_embedding_backward(dev, n, vocab, width, dtype, off):  # noqa: F811
    dt = DTYPES[dtype]
    lib = gf.load_library()
    dy = _randn(dev, n, width, seed=1, dtype=BF16)
    t = _randint(dev, -1, vocab + 1, n, seed=2)
    if n > 3:
        t[1], t[2], t[3] = vocab - 1, 0, vocab - 1
    g = Filled(dev, (vocab, width), dt, off)
    _call(dev, lib, lib.gefen_embedding_backward,
          lambda b: lib.gefen_embedding_backward_workspace(n, vocab, width, b),
          dy.data_ptr() if n else None, CODE[BF16], t.data_ptr() if n else None, 8, n, vocab, width,
          1.0, g.p, CODE[dt])
    g = g.check()
    on = t[(t >= 0) & (t < vocab)]
    used = torch.unique(on)
    if len(used):
        at = torch.searchsorted(used, t.clamp(0, vocab - 1)).clamp(max=len(used) - 1)
        at = torch.where((t >= 0) & (t < vocab), at, -1)
        want, size, count = _table_gradient(dy, at, len(used), 1.0)
        _within(g[used], want, (count + 1) * UNIT * size + HALF[dt] * (want.abs() + UNIT * size),
                "dtable")
    g[used] = 0
    assert not g.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 9, 9), (2, 50_257, 5), (700, 1003, 32),
                                            (2, 600_001, 20), (300, 300_001, 0)])
def test_token_logprobs(dev, rows, vocab, top, dtype):  # noqa: F811
    dt = DTYPES[dtype]
    lib = gf.load_library()
    z = _randn(dev, rows, vocab, seed=1, dtype=dt)
    t = _randint(dev, -1, vocab + 1, rows, seed=2)
    out = [Filled(dev, (rows,), F32) for _ in range(3)]
    best = [Filled(dev, (rows, top), d) for d in (F32, torch.int64)]
    _call(dev, lib, lib.gefen_token_logprobs,
          lambda b: lib.gefen_token_logprobs_workspace(CODE[dt], rows, vocab, top, b),
          z.data_ptr(), vocab, CODE[dt], rows, vocab, t.data_ptr(), 8, top, *(o.p for o in out),
          *(o.p for o in best))
    r = gf.token_logprobs(z, t, top=top)
    for got, want in zip(out + best, (r.logprob, r.entropy, r.lse, r.top_logprobs, r.top_tokens)):
        if want is not None:
            assert torch.equal(torch.nan_to_num(got.check(), nan=9.0), torch.nan_to_num(want, nan=9.0))
    assert torch.isfinite(r.lse).all() and (not top or (r.top_tokens >= 0).all())
    g, h = _randn(dev, rows, seed=3), _randn(dev, rows, seed=4)
    dz = Filled(dev, (rows, vocab), dt, 1)
    rc = lib.gefen_token_logprobs_backward(
        z.data_ptr(), vocab, CODE[dt], rows, vocab, t.data_ptr(), 8, r.lse.data_ptr(),
        r.entropy.data_ptr(), g.data_ptr(), h.data_ptr(), dz.p, vocab,
        torch.cuda.current_stream(dev).cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()
    want = gf.token_logprobs_backward(g, z, t, r.lse, r.entropy, dentropy=h)
    assert torch.equal(dz.check(), want) and torch.isfinite(want).all()


@pytest.mark.parametrize("n,width,vocab", [
    (1, 8, 5), (1, 512, 70_000), (1, 401, 20_000), (9, 513, 3001), (16, 2048, 1003), (17, 509, 1003),
    (64, 512, 1000), (130, 72, 2500), (256, 200, 3001), (257, 200, 3001), (1000, 765, 3001),
    (2100, 128, 6000), (4500, 64, 140_001)])
def test_head(dev, n, width, vocab):  # noqa: F811
    """(The last one's gradients of scores are taken by ranges of the vocabulary.)"""
    lib = gf.load_library()
    x = _randn(dev, n, width, seed=1, dtype=BF16)
    w = _randn(dev, vocab, width, seed=2).mul_(2 * width ** -0.5).to(BF16)
    t = _randint(dev, -1, vocab + 1, n, seed=3)
    out = [Filled(dev, (n,), F32) for _ in range(3)]
    _call(dev, lib, lib.gefen_head_logprobs,
          lambda b: lib.gefen_head_logprobs_workspace(n, width, vocab, 0, b),
          x.data_ptr(), w.data_ptr(), t.data_ptr(), 8, n, width, vocab, *(o.p for o in out))
    r = gf.head_logprobs(x, w, t)
    for got, want in zip(out, r):
        assert torch.equal(torch.nan_to_num(got.check(), nan=9.0), torch.nan_to_num(want, nan=9.0))
    assert torch.isfinite(r.lse).all() and torch.isfinite(r.entropy).all()
    g, h = _randn(dev, n, seed=4), _randn(dev, n, seed=5)
    want = gf.head_logprobs_backward(g, x, w, t, r.lse, r.entropy, dentropy=h)
    for which in ((True, True), (True, False), (False, True)):
        dx, dw = Filled(dev, (n, width), BF16), Filled(dev, (vocab, width), BF16)
        _call(dev, lib, lib.gefen_head_logprobs_backward,
              lambda b: lib.gefen_head_logprobs_workspace(n, width, vocab, 1, b),
              x.data_ptr(), w.data_ptr(), t.data_ptr(), 8, n, width, vocab, r.lse.data_ptr(),
              r.entropy.data_ptr(), g.data_ptr(), h.data_ptr(), dx.p if which[0] else None,
              dw.p if which[1] else None)
        for got, on, v in zip((dx, dw), which, want):
            if on:
                assert torch.equal(got.check(), v) and torch.isfinite(v).all()
            else:
                assert (got.bytes == 255).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 8, 1001])
def test_lookup_and_dropout(dev, n, dtype):  # noqa: F811
    dt = DTYPES[dtype]
    lib = gf.load_library()
    stream = torch.cuda.current_stream(dev).cuda_stream
    w = _randn(dev, 30, 77, seed=1, dtype=dt)
    t = _randint(dev, -1, 30, n, seed=2)
    y = Filled(dev, (n, 77), dt, 1)
    assert lib.gefen_embedding(t.data_ptr(), 8, n, w.data_ptr(), CODE[dt], 30, 77, 2.0, y.p, CODE[dt],
                               stream) == 0
    x = _randn(dev, n, seed=3, dtype=dt)
    d = Filled(dev, (n,), dt, 1)
    assert lib.gefen_dropout(x.data_ptr(), None, CODE[dt], n, 0.5, 3, 4, None, d.p, stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(y.check(), gf.embedding(t, w, scale=2.0))
    assert torch.equal(d.check(), gf.dropout(x, 0.5, 3, 4)) and torch.isfinite(d.t).all()
