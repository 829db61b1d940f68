"""The output head through each kernel that its plan can choose, against float64; the bounds are those
of test_gpu_language.py."""
import pytest
import torch

from head_sizes import SIZES
from test_gpu_language import (BF16, UNIT, _check_head_gradients, _check_rows, _head64, _randint,
                               _randn, dev)  # noqa: F401

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")


@pytest.mark.parametrize("n,width,vocab", SIZES)
def test_head(dev, n, width, vocab):  # noqa: F811
    x = _randn(dev, n, width, seed=1, dtype=BF16)
    w = _randn(dev, vocab, width, seed=2).mul_(2 * width ** -0.5).to(BF16)
    t = _randint(dev, -1, vocab, n, seed=3)
    g, h = _randn(dev, n, seed=4), _randn(dev, n, seed=5)
    r = gf.head_logprobs(x, w, t)
    _check_rows(r, _head64(x, w, t)[1])
    dx, dw = gf.head_logprobs_backward(g, x, w, t, r.lse, r.entropy, dentropy=h)
    _check_head_gradients(x, w, t, g, h, r, dx, dw)
    again = gf.head_logprobs_backward(g, x, w, t, r.lse, r.entropy, dentropy=h)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("n", [1, 2, 4, 16, 200])
def test_two_numbers_leave_the_outputs_own_rounding(dev, n):  # noqa: F811
    """Up to 256 tokens the scores' gradients are two bfloat16 numbers, together off by 2^-17 at
    most: what is left is the float32 sums' and the outputs' own rounding, checked against the
    formula with the kernel's lse and entropy."""
    width, vocab = 200, 1500
    x = _randn(dev, n, width, seed=1, dtype=BF16).double()
    w = _randn(dev, vocab, width, seed=2).mul_(2 * width ** -0.5).to(BF16).double()
    t = _randint(dev, 0, vocab, n, seed=3)
    g = _randn(dev, n, seed=4)
    r = gf.head_logprobs(x.to(BF16), w.to(BF16), t)
    dx, dw = gf.head_logprobs_backward(g, x.to(BF16), w.to(BF16), t, r.lse, r.entropy)
    d = x @ w.t() - r.lse.double()[:, None]
    p = d.exp()
    dz = -g.double()[:, None] * p
    # the score's own error (a float32 sum), the exponential's (with lse log2 e rounded), 2^-17
    err = width * UNIT * (x.abs() @ w.abs().t()).amax(1)[:, None]
    bound = dz.abs() * (2 * err + (4 * d.abs() + 2 * r.lse.double().abs()[:, None] + 16) * UNIT)
    dz[torch.arange(n, device=dev), t] += g.double()
    bound = bound + (2.0 ** -17 + 4 * UNIT) * (dz.abs() + bound) + 2.0 ** -126
    for got, want, size in ((dx, dz @ w, bound @ w.abs() + vocab * UNIT * (dz.abs() @ w.abs())),
                            (dw, dz.t() @ x,
                             bound.t() @ x.abs() + 2 * n * UNIT * (dz.abs().t() @ x.abs()))):
        over = (got.double() - want).abs() - size - 2.0 ** -8 * (want.abs() + size)
        assert over.max().item() <= 0.0
