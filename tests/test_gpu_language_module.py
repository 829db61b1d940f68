"""``FeedForward`` with dropout, and the example that trains tokens, on the device."""
import importlib.util
import os

import pytest
import torch

from test_gpu_language import BF16, F64, ROUND, _pieces, _randint, _randn, dev  # noqa: F401

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_feed_forward_with_dropout(dev):  # noqa: F811
    """y is the block's y with the elements of its own seed and offset dropped, the gradients those
    of that y, bit for bit; evaluation drops nothing."""
    torch.manual_seed(0)
    plain = gf.FeedForward(128, 192, device=dev)
    block = gf.FeedForward(128, 192, device=dev, dropout=0.25, seed=6)
    block.load_state_dict({**plain.state_dict(), "drop.state": block.drop.state})
    x = _randn(dev, 70, 128, seed=1, dtype=BF16).requires_grad_()
    r = _randn(dev, 70, 128, seed=2, dtype=BF16)
    up = _randn(dev, 70, 128, seed=3, dtype=BF16)
    for step in range(2):
        y, h = block(x, r)
        y0, h0 = plain(x, r)
        want = gf.dropout(y0.detach(), 0.25, 6, step)
        assert torch.equal(y, want) and torch.equal(h, h0)
        got = torch.autograd.grad((y, h), [x, *block.parameters()], (up, up))
        also = torch.autograd.grad((y0, h0), [x, *plain.parameters()],
                                   (gf.dropout(up, 0.25, 6, step), up))
        for a, b in zip(got, also):
            assert torch.equal(a, b)
    assert block.drop.state.tolist() == [6, 2]
    block.eval()
    assert torch.equal(block(x, r)[0], plain(x, r)[0])
    with torch.no_grad():
        block.train()
        assert torch.equal(block(x, r)[0], gf.dropout(plain(x, r)[0], 0.25, 6, 2))


def test_dropout_module_gradients(dev):  # noqa: F811
    drop = gf.Dropout(0.5, seed=1, device=dev)
    x, r = (_randn(dev, 40, 33, seed=i).requires_grad_() for i in (1, 2))
    keep = torch.from_numpy(_pieces(40 * 33, 1, 0) >= 32768).to(dev).view(40, 33)
    y = drop(x, r)
    assert torch.equal(y, torch.where(keep, x * 2, 0) + r)
    y.sum().backward()
    assert torch.equal(x.grad, keep * 2.0) and torch.equal(r.grad, torch.ones_like(r))
    a = drop(x.detach(), r)                      # a gradient of the residual alone
    a.sum().backward()
    assert torch.equal(r.grad, torch.full_like(r, 2.0))


def test_state_resumes(dev):  # noqa: F811
    """A saved state drops the same elements again."""
    drop = gf.Dropout(0.3, seed=8, device=dev)
    x = _randn(dev, 1000, seed=1)
    drop(x)
    saved = {k: v.clone() for k, v in drop.state_dict().items()}
    second = drop(x)
    other = gf.Dropout(0.3, device=dev)
    other.load_state_dict(saved)
    assert torch.equal(other(x), second) and other.state.tolist() == [8, 2]


@pytest.mark.parametrize("tied", [False, True])
def test_example(dev, tied):  # noqa: F811
    """It runs, and the scores that it stores for the alternatives agree with the head's but for
    their rounding to bfloat16: 2^-8 of scores of at most 64 here."""
    spec = importlib.util.spec_from_file_location(
        "train_tokens", os.path.join(ROOT, "examples", "train_tokens.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, off = example.main(["--vocab", "300", "--width", "64", "--inner", "128", "--length",
                                     "32", "--sequences", "4", "--steps", "3", "--layers", "1",
                                     *(["--tied"] if tied else [])])
    assert first == first and last == last       # not NaN
    assert off <= 64 * ROUND


def test_example_gradients(dev):  # noqa: F811
    """The model's gradients in evaluation mode against float64 autograd: each lies within the
    roundings on its way in the mean of squares, 12 to bfloat16 (rows, norms, projections, gradients)
    of 2^-8 at most, and those of the block's three 8-bit checkpoints. A group of 64 has a step of at
    most its largest magnitude / 63.75 (its codes reach 64 at least); a rounding is off by step /
    sqrt(12) in the mean of squares, and the largest of 64 values here is below 4 times their
    root mean square: 4 / 63.75 / sqrt(12) = 0.0182 each."""
    spec = importlib.util.spec_from_file_location(
        "train_tokens", os.path.join(ROOT, "examples", "train_tokens.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    torch.manual_seed(3)
    model = example.Model(200, 64, 128, 1, 0.1, False, dev).eval()
    t, nxt = _randint(dev, 0, 200, 64, seed=1), _randint(dev, -1, 200, 64, seed=2)
    logprob, entropy = model(t, nxt)
    (-logprob.mean() - 0.1 * entropy.mean()).backward()
    p = {n: v.detach().to(F64).requires_grad_() for n, v in model.named_parameters()}

    def norm(v, w):
        return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * w

    x = p["embed.table"][t] * model.embed.scale
    n = norm(x, p["blocks.0.norm"])
    a = torch.nn.functional.silu(n @ p["blocks.0.w_gate"].t()) * (n @ p["blocks.0.w_up"].t())
    x = x + a @ p["blocks.0.w_down"].t()
    lp = torch.log_softmax(norm(x, p["norm"]) @ p["head.weight"].t(), 1)
    taken = torch.where(nxt >= 0, lp.gather(1, nxt.clamp(min=0)[:, None])[:, 0], 0.0)
    (-taken.mean() + 0.1 * (lp.exp() * lp).sum(1).mean()).backward()
    for name, v in model.named_parameters():
        err = (v.grad.to(F64) - p[name].grad).norm() / p[name].grad.norm()
        assert err.item() <= (12 * ROUND ** 2 + 3 * 0.0182 ** 2) ** 0.5, (name, err.item())
