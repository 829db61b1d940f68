"""The Python layer of the feed-forward operators without a device: tensors of the host stand in for
device tensors, and the library is a recorder, so that what would be launched is seen and nothing
is."""
import pytest
import torch

import paper_2606_13894_amd as gf

ff = pytest.importorskip("paper_2606_13894_amd.feed_forward")

BF16, F32 = torch.bfloat16, torch.float32


class _On0(torch.Tensor):
    """A host tensor that says it is on device 0."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


class _On1(_On0):
    def get_device(self):
        return 1


def _tensor(where, *shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(where)


def _checkpoint(where, rows, cols):
    """As a call under that device would have made it."""
    c = gf.Checkpoint8.__new__(gf.Checkpoint8)
    c.codes = _tensor(where, rows, cols, dtype=torch.int8)
    c.exponents = _tensor(where, rows, -(-cols // 64), dtype=torch.uint8)
    return c


@pytest.fixture
def launched(monkeypatch):
    """The names of the entry points called; device 0 is the current one."""
    names = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: names.append(name) or 0

    monkeypatch.setattr(ff, "_library", Library)
    monkeypatch.setattr(ff, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return names


# ------------------------------------------------------------------ checkpoints of another device
def test_decode_takes_the_current_device_only(launched):
    _checkpoint(_On0, 3, 100).decode()
    assert launched == ["gefen_checkpoint_decode"]
    with pytest.raises(ValueError, match="current device"):
        _checkpoint(_On1, 3, 100).decode()
    assert launched == ["gefen_checkpoint_decode"]


def _norm_backward(saved):
    return gf.rms_norm_backward(_tensor(_On0, 3, 100), saved, _tensor(_On0, 3, dtype=F32),
                                _tensor(_On0, 100, dtype=F32))


def _ffn_backward(x, gate, up):
    w = _tensor(_On0, 40, 100)
    return gf.gated_ffn_backward(_tensor(_On0, 3, 100), x, (gate, up), w, w,
                                 _tensor(_On0, 100, 40))


def test_backward_takes_checkpoints_of_its_device_only(launched):
    here, there = _checkpoint(_On0, 3, 40), _checkpoint(_On1, 3, 40)
    x, far = _checkpoint(_On0, 3, 100), _checkpoint(_On1, 3, 100)
    _norm_backward(x)
    _ffn_backward(x, here, here)
    assert [n for n in launched if not n.endswith("workspace")] == [
        "gefen_rms_norm_backward", "gefen_gated_ffn_backward"]
    del launched[:]
    for call in (lambda: _norm_backward(far), lambda: _ffn_backward(far, here, here),
                 lambda: _ffn_backward(x, there, here), lambda: _ffn_backward(x, here, there)):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert launched == []
