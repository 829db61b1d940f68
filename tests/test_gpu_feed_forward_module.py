"""``FeedForward`` on the device outside training, and what it keeps."""
import pytest
import torch

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")
ff = pytest.importorskip("paper_2606_13894_amd.feed_forward")

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    return torch.device("cuda", 0)


def _rows(dev, T, K, seed):
    gen = torch.Generator(device=dev).manual_seed(seed)
    return torch.randn(T, K, generator=gen, device=dev).to(BF16)


# No gradient is wanted under no_grad, in inference mode, and where neither the inputs nor the
# parameters ask for one.
def _no_grad(block, *a):
    with torch.no_grad():
        return block(*a)


def _inference(block, *a):
    with torch.inference_mode():
        return block(*a)


def _frozen(block, *a):
    return block.requires_grad_(False)(*a)


@pytest.mark.parametrize("how", [_no_grad, _inference, _frozen])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [1, 9, 16, 17, 300])
def test_module_without_gradients_saves_nothing(dev, monkeypatch, T, act, residual, how):
    """The same outputs, and no checkpoint: beyond 16 tokens bit for bit, up to 16 within the
    roundings of A and y to bfloat16 (other kernels, another order of the sums)."""
    K, F = 200, 328
    torch.manual_seed(T)
    block = gf.FeedForward(K, F, activation=act, device=dev)
    x = _rows(dev, T, K, 1)
    r = _rows(dev, T, K, 2) if residual else None
    y, h = block(x, r)
    assert y.requires_grad

    def made(*a, **k):
        raise AssertionError("a checkpoint was made")

    monkeypatch.setattr(ff.Checkpoint8, "like", made)
    y1, h1 = how(block, x, r)
    assert not y1.requires_grad and torch.equal(h1, h) and h1.shape == x.shape
    if T > 16:
        assert torch.equal(y1, y)
    else:
        assert (y1.double() - y.double()).norm() <= 2 * 2.0 ** -8 * y.double().norm()


def test_everything_kept_for_the_backward_pass(dev):
    """Bytes an element in 8 bits, a float per row, and the bfloat16 copies of the weights that the
    call made; the norm's weight is the parameter itself."""
    T, K, F = 256, 512, 1024
    block = gf.FeedForward(K, F, device=dev)
    x = _rows(dev, T, K, 1).requires_grad_(True)
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (kept.append(t), t)[1], lambda t: t):
        block(x)
    own = [t for t in kept if t.data_ptr() != block.norm.data_ptr()]
    assert sum(t.numel() * t.element_size() for t in own) == \
        T * (K + K // 64 + 2 * (F + F // 64) + 4) + 3 * 2 * K * F


def test_gradients_that_are_not_there_are_errors(dev):
    """On the device as with stand-ins: under create_graph the gradients are the same bits, and
    going through them, or through a plain call's result, raises."""
    torch.manual_seed(0)
    block = gf.FeedForward(64, 96, device=dev)
    x = _rows(dev, 20, 64, 1).requires_grad_(True)
    (want,) = torch.autograd.grad(block(x)[0].sum(), x)
    (got,) = torch.autograd.grad(block(x)[0].sum(), x, create_graph=True)
    assert torch.equal(got, want) and not want.requires_grad
    with pytest.raises(RuntimeError, match="second derivative"):
        got.float().square().sum().backward()
    n = gf.rms_norm(x, block.norm)
    assert torch.equal(n.y, gf.rms_norm(x.detach(), block.norm.detach()).y)
    with pytest.raises(RuntimeError, match="FeedForward"):
        n.y.float().sum().backward()
    w = [p.detach().to(BF16) for p in (block.w_gate, block.w_up, block.w_down)]
    with pytest.raises(RuntimeError, match="FeedForward"):
        gf.gated_ffn(x, *w).float().sum().backward()
    assert not gf.gated_ffn(x.detach(), *w).requires_grad
