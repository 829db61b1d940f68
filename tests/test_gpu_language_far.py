"""Scores far from zero, as a finite mask over a whole row leaves them, against float64 formulas.

Bounds are those of ``test_gpu_language.py``: they grow with a score's distance d from the row's largest
one, not with the score itself, but for lse, which is rounded to float32. Where d is far above the sum's
logarithm, a log probability has up to four roundings of it (the difference, the products with log2 e and
ln 2, the logarithm's subtraction) and the two constants' own, 0.3 of one in all: 4.3 units of d, of which
those bounds have 3."""
import math

import pytest
import torch

from test_gpu_language import (BF16, DTYPES, F32, F64, HALF, UNIT, _check_rows,  # noqa: F401
                               _randint, _rows64, _within, dev)

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")

LEVELS = [3e4, 1e5, 2.0 ** 20 - 1, 2.0 ** 20, 1.3e6, 1e8, 1e9, 3e9, 1e10, 7e14, 1e20, 1e30, 8e37, 9e37,
          3e38]


def _rows(z, t):
    want = _rows64(z, t)
    more = 2 * UNIT * torch.nan_to_num(want["d"].abs(), posinf=0.0)
    want["b_lp"] = want["b_lp"] + more
    want["b_logprob"] = want["b_logprob"] + more.gather(1, t.clamp(min=0)[:, None])[:, 0]
    return want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(30, 777), (30, 50257), (600, 1003), (60, 300_001)])
def test_rows_at_one_level(dev, rows, vocab, dtype):  # noqa: F811
    """A row whose scores are all masked by the same finite number, or lie a few steps of its type
    around it: what counts is their differences."""
    dt = DTYPES[dtype]
    z = torch.empty(rows, vocab, dtype=dt, device=dev)
    step = _randint(dev, 0, 4, vocab, seed=1)
    for r in range(rows):
        v = torch.tensor(LEVELS[r // 2 % len(LEVELS)] * (-1) ** r, dtype=dt)
        levels = [v]
        for _ in range(3):                       # the next numbers of the type
            levels.append(torch.nextafter(levels[-1], torch.zeros_like(v)))
        z[r] = torch.stack(levels).to(dev)[step] if r % 4 < 2 else v
    t = _randint(dev, 0, vocab, rows, seed=2)
    want = _rows(z, t)
    for top in (0, 4):
        _check_rows(gf.token_logprobs(z, t, top=top), want, top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("rows,vocab", [(3, 4000), (700, 4000), (2, 400_000)])
def test_levels_among_lanes(dev, rows, vocab, sign, dtype):  # noqa: F811
    """Scores around 2^20, on both sides of which the sums take different forms, so that lanes, waves and
    parts of a row differ in theirs; and rows whose scores grow or fall along the row."""
    z = sign * (2.0 ** 20 + torch.randint(-6, 7, (rows, vocab), device=dev,
                                          generator=torch.Generator(dev).manual_seed(1)).to(F32))
    z = z.to(DTYPES[dtype])
    ramp = torch.linspace(-2e6, 2e6, vocab, device=dev).to(DTYPES[dtype])
    z[0], z[1] = ramp, ramp.flip(0)
    t = _randint(dev, 0, vocab, rows, seed=2)
    t[:2] = torch.tensor([vocab - 1, 5], device=dev)
    _check_rows(gf.token_logprobs(z, t, top=3), _rows(z, t), 3)


@pytest.mark.parametrize("n,vocab,width", [(1, 1003, 64), (9, 1003, 64), (16, 999, 61), (64, 1000, 128),
                                           (1, 70_000, 64), (300, 4097, 256), (1000, 6000, 64)])
@pytest.mark.parametrize("sign", [1, -1])
def test_head_at_one_level(dev, n, vocab, width, sign):  # noqa: F811
    """Every score is the same number of about 10^13 (exactly: 1.25 times a power of two times the width), or, in
    odd rows, 2^-20 of it."""
    x = torch.full((n, width), sign * 1.25 * 2.0 ** 18, dtype=BF16, device=dev)
    x[1::2] = sign * 1.25 * 2.0 ** -2
    w = torch.full((vocab, width), 2.0 ** 19, dtype=BF16, device=dev)
    t = _randint(dev, 0, vocab, n, seed=1)
    r = gf.head_logprobs(x, w, t)
    size = torch.where(torch.arange(n, device=dev) % 2 == 0, 1.25 * 2.0 ** 37, 1.25 * 2.0 ** 17).to(F64)
    lse = sign * width * size + math.log(vocab)
    log = torch.full((n,), math.log(vocab), dtype=F64, device=dev)
    bound = (vocab / 256 + 64 + 16) * UNIT * (1 + log)
    _within(r.logprob, -log, bound, "logprob")
    _within(r.entropy, log, bound, "entropy")
    _within(r.lse, lse, bound + UNIT * lse.abs(), "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(6, 40), (6, 50257), (700, 1003), (6, 600_001)])
def test_the_lowest_number_among_others(dev, rows, vocab, dtype):  # noqa: F811
    """Rows of ordinary scores, some masked by the type's lowest number (or a little less): the log
    probability of a masked token is z - lse, not -inf, also among the alternatives where fewer scores
    than these are left. (Rows 2 and 3: among scores of 10^38, below which it may pass the type's range.)"""
    dt = DTYPES[dtype]
    low = torch.finfo(dt).min
    z = torch.randn(rows, vocab, generator=torch.Generator(dev).manual_seed(1), device=dev).to(dt)
    gone = torch.rand(rows, vocab, generator=torch.Generator(dev).manual_seed(2), device=dev) < 0.5
    z[gone] = low
    z[1] = low
    z[1, :3] = torch.tensor([1.0, -2.0, 0.5], dtype=dt)          # three left
    z[2] = -2e38
    z[2, 7] = 1e38
    z[3] = low
    z[3, 7] = 3e38
    z[4] = -2.5e38
    z[4, ::2] = low
    z[4, 9] = -1e6
    t = _randint(dev, 0, vocab, rows, seed=3)
    t[:6] = torch.tensor([gone[0].nonzero()[0, 0].item(), 20, 8, 8, 10, -1], device=dev)
    want = _rows(z, t)
    assert torch.isfinite(want["logprob"][[0, 1, 2, 4]]).all()
    for top in (0, 6, 32):
        _check_rows(gf.token_logprobs(z, t, top=top), want, top)


@pytest.mark.parametrize("n,vocab,width", [(1, 1003, 64), (9, 1003, 64), (16, 999, 61), (64, 1000, 128),
                                           (1, 70_000, 64), (300, 4097, 256)])
def test_head_of_a_score_far_below(dev, n, vocab, width):  # noqa: F811
    """Every second weight row gives scores of -3 * 2^126 (two terms, exactly), the others 0."""
    x = torch.zeros(n, width, dtype=BF16, device=dev)
    x[:, :2] = 2.0 ** 63
    w = torch.zeros(vocab, width, dtype=BF16, device=dev)
    w[1::2, :2] = -1.5 * 2.0 ** 63
    t = torch.ones(n, dtype=torch.int64, device=dev)
    t[1::2] = 2
    r = gf.head_logprobs(x, w, t)
    lse = math.log((vocab + 1) // 2)
    want = torch.where(t == 1, -3.0 * 2.0 ** 126, 0.0).to(F64) - lse
    bound = (vocab / 256 + 64 + 16) * UNIT * (1 + lse)
    _within(r.logprob, want, bound + 2 * UNIT * want.abs(), "logprob")


def _gradient(z, t, g, h):
    """The float64 gradient of the scores, from the scores alone, and its bound before the output's
    rounding. p is off by what its exponent is off by, (4 |log p| + 8) units (as in the sums) and the logarithm
    of the sum's bound, which the entropy's holds; values below 2^-126 may be flushed before their factor."""
    w = _rows64(z, t)
    V = z.shape[1]
    g, h, H, err = (v.to(F64)[:, None] for v in (g, h, w["H"], w["b_H"]))
    on = ((t >= 0) & (t < V))[:, None]
    g = torch.where(on, g, 0.0)
    lp = torch.where(w["p"] > 0, w["lp"], 0.0)
    hit = torch.zeros_like(w["p"]).scatter_(1, t.clamp(0, V - 1)[:, None], 1.0) * on
    inner = lp + H
    want = hit * g - w["p"] * (g + h * inner)
    size = g.abs() + h.abs() * inner.abs()
    bound = w["p"] * (size * ((4 * lp.abs() + 16) * UNIT + err)
                      + h.abs() * (2 * err + 4 * UNIT * (lp.abs() + H.abs())))
    return want, bound + hit * 2 * UNIT * g.abs() + 2.0 ** -126 * (1 + g.abs() + 120 * h.abs())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(40, 7), (40, 1003), (40, 50257), (40, 300_001)])
def test_gradients_of_the_module(dev, rows, vocab, dtype):  # noqa: F811
    """Rows at one level, some of their scores a few steps of the type lower, the lowest number among
    others, large scores, ordinary ones and empty rows: the gradients are the formula's, whatever lse is."""
    dt = DTYPES[dtype]
    gen = torch.Generator(dev).manual_seed(1)
    z = torch.randn(rows, vocab, generator=gen, device=dev)
    z[35:39] *= torch.tensor([1e2, 1e4, 1e6, 1e9], device=dev)[:, None]
    z = z.to(dt)
    step = _randint(dev, 0, 3, vocab, seed=1)
    for r in range(30):
        v = torch.tensor(LEVELS[r // 2] * (-1) ** r, dtype=dt)
        levels = [v]
        for _ in range(2):
            levels.append(torch.nextafter(levels[-1], torch.zeros_like(v)))
        z[r] = torch.stack(levels).to(dev)[step] if r % 4 < 2 else v
    z[30] = torch.finfo(dt).min
    z[31, ::2] = torch.finfo(dt).min
    z[32, 1::2] = -1e9
    z[33] = -math.inf
    t = _randint(dev, -1, vocab + 1, rows, seed=2)
    g, h = (torch.randn(rows, generator=gen, device=dev) for _ in range(2))
    leaf = z.clone().requires_grad_()
    logprob, entropy = gf.LogProbs()(leaf, t)
    torch.autograd.backward((logprob, entropy), (g, h))
    want, bound = _gradient(z, t, g, h)
    want[33], bound[33] = 0.0, 0.0
    _within(leaf.grad, want, bound + HALF[dt] * want.abs(), "dlogits")
    plain = gf.token_logprobs(z, t)
    assert torch.equal(torch.nan_to_num(logprob), torch.nan_to_num(plain.logprob))
    assert torch.equal(entropy, plain.entropy)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,top", [(3, 9, 4), (700, 1003, 0), (2, 600_001, 20)])
def test_lse_in_two_numbers(dev, rows, vocab, top, dtype):  # noqa: F811
    """Their sum is closer to lse than one number can be; the other results are those of the plain entry."""
    from test_gpu_language_written import CODE, Filled, _call
    dt = DTYPES[dtype]
    lib = gf.load_library()
    z = (torch.randn(rows, vocab, generator=torch.Generator(dev).manual_seed(1), device=dev)
         * 3 + 1000).to(dt)
    z[0] = -3e4
    z[1] = -math.inf
    z[2 % rows, 5] = math.nan if rows > 2 else 1.0
    t = _randint(dev, -1, vocab + 1, rows, seed=2)
    out = [Filled(dev, (rows,), F32) for _ in range(4)]
    best = [Filled(dev, (rows, top), d) for d in (F32, torch.int64)]
    _call(dev, lib, lib.gefen_token_logprobs_split,
          lambda b: lib.gefen_token_logprobs_workspace(CODE[dt], rows, vocab, top, b),
          z.data_ptr(), vocab, CODE[dt], rows, vocab, t.data_ptr(), 8, top, *(o.p for o in out),
          *(o.p for o in best))
    logprob, entropy, lse, rest = (o.check() for o in out)
    r = gf.token_logprobs(z, t, top=top)
    for got, want in ((logprob, r.logprob), (entropy, r.entropy), (lse, r.lse),
                      (best[0].check(), r.top_logprobs), (best[1].check(), r.top_tokens)):
        if want is not None:
            assert torch.equal(torch.nan_to_num(got, nan=9.0), torch.nan_to_num(want, nan=9.0))
    want = _rows64(z, t)
    fine = torch.isfinite(r.lse)
    assert (rest[~fine] == 0).all() and fine.any() and not fine.all()
    # b_H holds the logarithm's bound; the sum of the two is off by that alone
    both = (lse.to(F64) + rest.to(F64))[fine]
    assert ((both - want["lse"][fine]).abs() <= want["b_H"][fine] + 2.0 ** -40).all()
