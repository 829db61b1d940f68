"""Every kernel of the gated block that the plan can choose, against the float64 formulas term by
term (the bounds are those of test_gpu_feed_forward.py): the larger tiles with sums of few and of
many stages, split and unsplit, and the few-token kernels at each number of rows and waves.

Beside those bounds, which grow with a sum's length, each output as a whole: two roundings to
bfloat16 lie between it and the formula, of the product's operand and of the output, each at most
2^-9 of a value, and independent from term to term, so that the first moves a sum by no more of
its norm than of a term: 2^-8 of the norm in all. (One term too few in a sum of n moves it by about
n^(-1/2), 0.01 for the longest sum here.)"""
import pytest
import torch

from ffn_sizes import FEW, TILES
from test_gpu_feed_forward import (F64, _act64, _check_backward, _check_forward, _decode64,
                                   _ffn_inputs, _randn, _slope64)

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    return torch.device("cuda", 0)


def _near(got, want, what):
    assert (got.to(F64) - want).norm() <= 2.0 ** -8 * want.norm(), what


def _forward64(x, wg, wu, wd, act):
    x, wg, wu, wd = (t.to(F64) for t in (x, wg, wu, wd))
    return (_act64(x @ wg.t(), act) * (x @ wu.t())) @ wd.t()


def _backward64(dy, xs, saved, wg, wu, wd, act, gain):
    dy, wg, wu, wd = (t.to(F64) for t in (dy, wg, wu, wd))
    g, u = _decode64(saved[0]), _decode64(saved[1])
    da, a = dy @ wd, _act64(g, act)
    dg, du = da * u * _slope64(g, act), da * a
    by = 1.0 if gain is None else gain.to(F64)
    return dg @ wg + du @ wu, (dg.t() @ xs) * by, (du.t() @ xs) * by, dy.t() @ (a * u)


@pytest.mark.parametrize("T,K,F", TILES)
def test_tiles(dev, T, K, F):
    act = "gelu" if (T + K + F) % 2 else "silu"
    x, wg, wu, wd, dy = _ffn_inputs(dev, T, K, F, seed=T)
    y, saved = gf.gated_ffn(x, wg, wu, wd, activation=act, checkpoint=True)
    _check_forward(x, wg, wu, wd, act, y, saved)
    _near(y, _forward64(x, wg, wu, wd, act), "y")
    gain = 1 + 0.3 * _randn(dev, K, seed=99)
    xc = gf.checkpoint8(x)
    for keep, xs, by in ((x, x.to(F64), None), (xc, _decode64(xc), gain)):
        grads = gf.gated_ffn_backward(dy, keep, saved, wg, wu, wd, activation=act, gain=by)
        _check_backward(dy, xs, saved, wg, wu, wd, act, grads, by)
        for got, want, what in zip(grads, _backward64(dy, xs, saved, wg, wu, wd, act, by),
                                   ("dx", "dw_gate", "dw_up", "dw_down")):
            _near(got, want, what)
    again = gf.gated_ffn_backward(dy, xc, saved, wg, wu, wd, activation=act, gain=gain)
    assert all(torch.equal(p, q) for p, q in zip(grads, again))


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,K,F", FEW)
def test_few_tokens(dev, T, K, F, act):
    x, wg, wu, wd, _ = _ffn_inputs(dev, T, K, F, seed=T)
    y = gf.gated_ffn(x, wg, wu, wd, activation=act)
    _check_forward(x, wg, wu, wd, act, y, None)
    _near(y, _forward64(x, wg, wu, wd, act), "y")
    assert torch.equal(y, gf.gated_ffn(x, wg, wu, wd, activation=act))
