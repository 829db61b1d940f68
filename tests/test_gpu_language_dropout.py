"""The ``Dropout`` module's numbers on the device."""
import pytest
import torch

from test_gpu_language import BF16, _dropped, _pieces, _randn, dev  # noqa: F401

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")


def test_default_modules_drop_different_elements(dev):  # noqa: F811
    """A stack of blocks made without seeds: no two of them share their zeros, and p is kept to."""
    torch.manual_seed(1)
    drops = [gf.Dropout(0.5, device=dev) for _ in range(3)]
    drops += [gf.FeedForward(64, 64, device=dev, dropout=0.5).drop for _ in range(3)]
    x = torch.ones(1 << 16, device=dev)
    zeros = [drop(x) == 0 for drop in drops]
    for i, a in enumerate(zeros):
        seed, at = drops[i].state.tolist()
        assert at == 1 and torch.equal(drops[i](x), gf.dropout(x, 0.5, seed, 1))
        for b in zeros[:i]:
            # independent ones agree on half of 2^16 elements, with a deviation of 128
            assert abs((a == b).sum().item() - (1 << 15)) < 8 * 128


def test_first_pass_in_a_graph(dev):  # noqa: F811
    """Without a pass before the capture the seed is drawn by the first replay, or by an eager pass before
    it; a state that is loaded later is not touched."""
    torch.manual_seed(2)
    x = _randn(dev, 40, 64, seed=1, dtype=BF16)
    for eager_first in (False, True):
        drop = gf.Dropout(0.25, device=dev)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = drop(x)
        assert drop.state.tolist() == [0, 0]
        at = 0
        if eager_first:
            drop(x)
            at = 1
        for _ in range(3):
            graph.replay()
            seed, now = drop.state.tolist()
            assert seed > 0 and now == at + 1
            assert torch.equal(y, _dropped(x, 0.25, _pieces(x.numel(), seed, at).reshape(-1)))
            at += 1
            z = drop(x)
            assert torch.equal(z, gf.dropout(x, 0.25, seed, at))
            at += 1
        drop.load_state_dict({"state": torch.tensor([77, 5])})
        graph.replay()
        assert torch.equal(y, gf.dropout(x, 0.25, 77, 5)) and drop.state.tolist() == [77, 6]


@pytest.mark.parametrize("reentrant", [False, True])
def test_recomputed_blocks(dev, reentrant):  # noqa: F811
    """Activations that are computed again: an error with dropout, the same gradients without."""
    from torch.utils.checkpoint import checkpoint
    torch.manual_seed(3)
    block = gf.FeedForward(64, 128, device=dev)
    x = _randn(dev, 20, 64, seed=1, dtype=BF16).requires_grad_()
    up = _randn(dev, 20, 64, seed=2, dtype=BF16)
    inputs = [x, *block.parameters()]
    for v in inputs:
        v.grad = None
    torch.autograd.backward(block(x)[0], up)
    want = [v.grad.clone() for v in inputs]
    for v in inputs:
        v.grad = None
    torch.autograd.backward(checkpoint(block, x, use_reentrant=reentrant)[0], up)
    assert all(torch.equal(v.grad, w) for v, w in zip(inputs, want))
    dropping = gf.FeedForward(64, 128, device=dev, dropout=0.1)
    y, _ = checkpoint(dropping, x, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="run again within a backward pass"):
        torch.autograd.backward(y, up)
