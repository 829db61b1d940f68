"""A checkpoint of more elements than a launch has threads for (2^35 elements are 2^32 vectors)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")

BF16 = torch.bfloat16


def test_checkpoint_past_a_launch(dev_memory=100 << 30):
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < dev_memory:
        pytest.skip("needs 100 GiB of device memory")
    dev = torch.device("cuda", 0)
    groups = (1 << 29) + 3                         # 2^35 + 192 elements, one to a row here
    ends = [k << 27 for k in range(1, 5)]          # launches end at multiples of 2^28 groups
    at = sorted({0, 1, groups - 1, groups - 3, *(e + d for e in ends for d in (-1, 0, 1))})
    gen = torch.Generator(device=dev).manual_seed(1)
    some = torch.randn(len(at), 64, generator=gen, device=dev).to(BF16)
    rows = torch.tensor(at, device=dev)
    x = torch.zeros(groups, 64, dtype=BF16, device=dev)
    x[rows] = some
    c, alone = gf.checkpoint8(x), gf.checkpoint8(some)
    assert torch.equal(c.codes[rows], alone.codes)
    assert torch.equal(c.exponents[rows], alone.exponents)
    others = c.exponents.view(-1) != 1             # a group of zeros has the smallest exponent
    assert others.sum().item() == len(at) and others[rows].all()
    del others
    x.fill_(1.0)
    c.decode(out=x)
    assert torch.equal(x[rows], alone.decode())
    x[rows] = 0.0
    assert not any(part.any().item() for part in x.split(1 << 24))
    del x, c
    torch.cuda.empty_cache()
