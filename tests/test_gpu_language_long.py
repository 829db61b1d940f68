"""The operators at a language model's two ends where offsets pass 32 bits: tables, rows of scores and
outputs of more than 2^32 bytes and elements, dropout of more than 2^35 elements."""
import ctypes

import pytest
import torch

from test_gpu_language import BF16, F64, ROUND, UNIT, _dropped, _pieces, _randint, _randn, dev  # noqa: F401

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")


def _room(gib):
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def test_embedding_of_a_long_table(dev):  # noqa: F811
    _room(40)
    vocab, width = (1 << 21) + 7, 2056               # 4.3e9 elements
    w = torch.empty(vocab, width, dtype=BF16, device=dev)
    last = torch.tensor([vocab - 1, 0, vocab - 2, 2_090_000, vocab - 1, -1, 1_044_496],
                        device=dev)
    rows = _randn(dev, 7, width, seed=1, dtype=BF16)
    for i in (0, 1, 2, 3, 6):
        w[last[i]] = rows[i]
    y = gf.embedding(last, w)
    for i in (0, 1, 2, 3, 6):
        assert torch.equal(y[i], rows[i])
    assert torch.equal(y[4], rows[0]) and not y[5].any()
    del w, y
    dy = _randn(dev, 7, width, seed=2, dtype=BF16)
    g = gf.embedding_backward(dy, last, vocab, dtype=BF16)
    assert torch.equal(g[vocab - 1], (dy[0].float() + dy[4].float()).to(BF16))
    for i in (1, 2, 3, 6):
        assert torch.equal(g[last[i]], dy[i])
        g[last[i]] = 0
    g[vocab - 1] = 0
    for a in range(0, vocab, 1 << 18):
        assert not g[a:a + (1 << 18)].any()


def test_many_rows_of_scores(dev):  # noqa: F811
    _room(40)
    rows, vocab = 34_000, 128_256                    # 4.4e9 elements
    z = torch.empty(rows, vocab, dtype=BF16, device=dev)
    part = _randn(dev, 100, vocab, seed=1, dtype=BF16)
    z[:] = -1.0
    z[-100:] = part
    t = _randint(dev, 0, vocab, rows, seed=2)
    r = gf.token_logprobs(z, t, top=3)
    want = gf.token_logprobs(z[-600:].clone(), t[-600:], top=3)
    for a, b in zip(r, want):
        assert torch.equal(a[-600:], b)
    g = _randn(dev, rows, seed=3)
    own = gf.token_logprobs_backward(g[-100:], part, t[-100:], r.lse[-100:], r.entropy[-100:])
    gf.token_logprobs_backward(g, z, t, r.lse, r.entropy, out=z)
    assert torch.equal(z[-100:], own)


def test_dropout_of_many_elements(dev):  # noqa: F811
    """2^35 + 2^13 elements in place: the block's number passes 32 bits."""
    _room(70)
    n = (1 << 35) + (1 << 13)
    x = torch.ones(n, dtype=BF16, device=dev)
    lib = gf.load_library()
    stream = torch.cuda.current_stream(dev).cuda_stream
    assert lib.gefen_dropout(x.data_ptr(), None, 1, n, 0.25, 77, 5, None, x.data_ptr(),
                             stream) == 0
    for first in (0, 1 << 20, (1 << 31) - 4096, (1 << 32) - 4096, (1 << 34) + 8, (1 << 35) - 4096):
        part = x[first:first + 8192]
        assert torch.equal(part, _dropped(torch.ones_like(part), 0.25,
                                          _pieces(8192, 77, 5, first=first))), first


def test_head_of_a_long_weight(dev):  # noqa: F811
    """A weight of 2^32 elements and more, in ranges of the vocabulary; its gradient row by row where
    it is looked at."""
    _room(60)
    n, width, vocab = 20, 2048, (1 << 21) + 300
    w = torch.empty(vocab, width, dtype=BF16, device=dev)
    gen = torch.Generator(device=dev).manual_seed(1)
    for a in range(0, vocab, 1 << 18):
        b = min(vocab, a + (1 << 18))
        w[a:b] = torch.randn(b - a, width, generator=gen, device=dev).mul_(2 * width ** -0.5)
    x = _randn(dev, n, width, seed=2, dtype=BF16)
    t = torch.cat([torch.tensor([vocab - 1, 0, 1 << 20, (1 << 20) - 1], device=dev),
                   _randint(dev, 0, vocab, n - 4, seed=3)])
    g = _randn(dev, n, seed=4)
    r = gf.head_logprobs(x, w, t)
    x64 = x.to(F64)
    total = torch.zeros(n, dtype=F64, device=dev)
    for a in range(0, vocab, 1 << 18):
        total += (x64 @ w[a:a + (1 << 18)].to(F64).t()).exp().sum(1)
    lse = total.log()
    # the scores' error, the sums' (a tile's 32 terms a lane, 16400 slots) and the last rounding
    err = width * UNIT * (x64.abs() @ w[:1000].to(F64).abs().t()).amax(1) * 2
    assert ((r.lse.to(F64) - lse).abs() <= err + (64 + 16400 / 64 + 40) * UNIT + UNIT * lse).all()
    dx, dw = gf.head_logprobs_backward(g, x, w, t, r.lse, r.entropy)
    ex = torch.zeros(n, width, dtype=F64, device=dev)
    bx = torch.zeros_like(ex)
    for a in range(0, vocab, 1 << 18):
        wp = w[a:a + (1 << 18)].to(F64)
        d = x64 @ wp.t() - r.lse.to(F64)[:, None]
        dz = -g.to(F64)[:, None] * d.exp()
        bound = dz.abs() * (2 * err[:, None] + (4 * d.abs() + 64) * UNIT)
        rows = ((t >= a) & (t < a + wp.shape[0])).nonzero()[:, 0]
        dz[rows, t[rows] - a] += g.to(F64)[rows]
        bound = bound + (2.0 ** -17 + 4 * UNIT) * (dz.abs() + bound) + 2.0 ** -126
        ew = dz.t() @ x64
        bw = bound.t() @ x64.abs() + 2 * n * UNIT * (dz.abs().t() @ x64.abs())
        over = (dw[a:a + (1 << 18)].to(F64) - ew).abs() - bw - ROUND * (ew.abs() + bw)
        assert over.max().item() <= 0.0, a
        ex += dz @ wp
        bx += bound @ wp.abs() + vocab * UNIT * (dz.abs() @ wp.abs())
    assert ((dx.to(F64) - ex).abs() <= bx + ROUND * (ex.abs() + bx)).all()
