"""The Python layer of the operators at a language model's two ends without a device: tensors of the
host stand in for device tensors, and the library is a recorder, so that what would be launched is
seen and nothing is."""
import ctypes
import math

import pytest
import torch

import paper_2606_13894_amd as gf

ff = pytest.importorskip("paper_2606_13894_amd.feed_forward")
lm = pytest.importorskip("paper_2606_13894_amd.language")

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


def _ids(where, *shape, dtype=torch.int64):
    return _tensor(where, *shape, dtype=dtype)


@pytest.fixture
def calls(monkeypatch):
    """(name, arguments) of the entry points called; device 0 is the current one."""
    made = []

    class Library:
        def __getattr__(self, name):
            def entry(*a):
                if not name.endswith("workspace"):
                    made.append((name, a))
                return 0
            return entry

    lib = Library()
    monkeypatch.setattr(ff, "_library", lambda: lib)
    monkeypatch.setattr(ff, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(ff, "_current_device", lambda: 0)
    return made


def _embedding(t=None, w=None):
    return gf.embedding(_ids(_On0, 3) if t is None else t, _tensor(_On0, 9, 8) if w is None else w)


def _embedding_backward(dy=None, t=None):
    return gf.embedding_backward(_tensor(_On0, 3, 8) if dy is None else dy,
                                 _ids(_On0, 3) if t is None else t, 9)


def _dropout(x=None, seed=1, r=None):
    return gf.dropout(_tensor(_On0, 3, 8) if x is None else x, 0.1, seed, residual=r)


def _scores(z=None, t=None):
    return gf.token_logprobs(_tensor(_On0, 3, 8) if z is None else z,
                             _ids(_On0, 3) if t is None else t)


def _scores_backward(g=None, z=None, t=None, lse=None, ent=None, h=None, out=None):
    f = _tensor(_On0, 3, dtype=F32)
    return gf.token_logprobs_backward(
        f if g is None else g, _tensor(_On0, 3, 8) if z is None else z,
        _ids(_On0, 3) if t is None else t, f if lse is None else lse, f if ent is None else ent,
        dentropy=h, out=out)


def _head(x=None, w=None, t=None):
    return gf.head_logprobs(_tensor(_On0, 3, 8) if x is None else x,
                            _tensor(_On0, 9, 8) if w is None else w,
                            _ids(_On0, 3) if t is None else t)


def _head_backward(g=None, x=None, w=None, t=None, lse=None, ent=None, h=None):
    f = _tensor(_On0, 3, dtype=F32)
    return gf.head_logprobs_backward(
        f if g is None else g, _tensor(_On0, 3, 8) if x is None else x,
        _tensor(_On0, 9, 8) if w is None else w, _ids(_On0, 3) if t is None else t,
        f if lse is None else lse, f if ent is None else ent, dentropy=h)


F1 = _tensor(_On1, 3, dtype=F32)


@pytest.mark.parametrize("call,arguments", [
    (_embedding, dict(t=_ids(_On1, 3))), (_embedding, dict(w=_tensor(_On1, 9, 8))),
    (_embedding_backward, dict(dy=_tensor(_On1, 3, 8))),
    (_embedding_backward, dict(t=_ids(_On1, 3))),
    (_dropout, dict(x=_tensor(_On1, 3, 8))), (_dropout, dict(r=_tensor(_On1, 3, 8))),
    (_dropout, dict(seed=_ids(_On1, 2))),
    (_scores, dict(z=_tensor(_On1, 3, 8))), (_scores, dict(t=_ids(_On1, 3))),
    (_scores_backward, dict(g=F1)), (_scores_backward, dict(z=_tensor(_On1, 3, 8))),
    (_scores_backward, dict(t=_ids(_On1, 3))), (_scores_backward, dict(lse=F1)),
    (_scores_backward, dict(ent=F1)), (_scores_backward, dict(h=F1)),
    (_scores_backward, dict(out=_tensor(_On1, 3, 8))),
    (_head, dict(x=_tensor(_On1, 3, 8))), (_head, dict(w=_tensor(_On1, 9, 8))),
    (_head, dict(t=_ids(_On1, 3))),
    (_head_backward, dict(g=F1)), (_head_backward, dict(x=_tensor(_On1, 3, 8))),
    (_head_backward, dict(w=_tensor(_On1, 9, 8))), (_head_backward, dict(t=_ids(_On1, 3))),
    (_head_backward, dict(lse=F1)), (_head_backward, dict(ent=F1)), (_head_backward, dict(h=F1)),
])
def test_tensors_of_the_current_device_only(calls, call, arguments):
    call()
    assert len(calls) == 1
    with pytest.raises(ValueError, match="current device"):
        call(**arguments)
    assert len(calls) == 1


def _plain(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype)


@pytest.mark.parametrize("call", [
    lambda: _embedding(t=_plain(3, dtype=torch.int64)), lambda: _embedding(w=_plain(9, 8)),
    lambda: _embedding(t=[1, 2]), lambda: _dropout(x=_plain(3, 8)),
    lambda: _scores(z=_plain(3, 8)), lambda: _scores(t=_plain(3, dtype=torch.int64)),
    lambda: _head(w=_plain(9, 8)), lambda: _head(t=None, x=_plain(3, 8)),
    lambda: _scores_backward(g=_plain(3, dtype=F32)),
])
def test_host_tensors_are_refused(calls, call):
    with pytest.raises(ValueError, match="device tensor"):
        call()
    assert calls == []


@pytest.mark.parametrize("error,call", [
    (TypeError, lambda: _embedding(t=_tensor(_On0, 3, dtype=torch.int16))),
    (TypeError, lambda: _embedding(t=_tensor(_On0, 3, dtype=F32))),
    (TypeError, lambda: _embedding(w=_tensor(_On0, 9, 8, dtype=torch.float16))),
    (ValueError, lambda: _embedding(w=_tensor(_On0, 72))),
    (ValueError, lambda: _embedding(w=_tensor(_On0, 0, 8))),
    (ValueError, lambda: _embedding(w=_tensor(_On0, 9, 0))),
    (TypeError, lambda: gf.embedding(_ids(_On0, 3), _tensor(_On0, 9, 8), dtype=torch.float16)),
    (ValueError, lambda: _embedding_backward(t=_ids(_On0, 4))),
    (ValueError, lambda: gf.embedding_backward(_tensor(_On0, 3, 8), _ids(_On0, 3), 0)),
    (TypeError, lambda: gf.embedding_backward(_tensor(_On0, 3, 8), _ids(_On0, 3), 9,
                                              dtype=torch.float64)),
    (TypeError, lambda: _dropout(x=_tensor(_On0, 3, 8, dtype=torch.float64))),
    (TypeError, lambda: _dropout(r=_tensor(_On0, 3, 8, dtype=F32))),
    (ValueError, lambda: _dropout(r=_tensor(_On0, 8))),
    (TypeError, lambda: _dropout(seed=_tensor(_On0, 2, dtype=torch.int32))),
    (ValueError, lambda: _dropout(seed=_ids(_On0, 3))),
    (TypeError, lambda: _dropout(seed=1.5)),
    (ValueError, lambda: _scores(t=_ids(_On0, 4))),
    (ValueError, lambda: _scores(z=_tensor(_On0, 3, 0))),
    (TypeError, lambda: _scores(z=_tensor(_On0, 3, 8, dtype=torch.float16))),
    (ValueError, lambda: gf.token_logprobs(_tensor(_On0, 3, 8), _ids(_On0, 3), top=9)),
    (ValueError, lambda: gf.token_logprobs(_tensor(_On0, 3, 80), _ids(_On0, 3), top=33)),
    (ValueError, lambda: gf.token_logprobs(_tensor(_On0, 3, 8), _ids(_On0, 3), top=-1)),
    (TypeError, lambda: _scores_backward(g=_tensor(_On0, 3))),
    (ValueError, lambda: _scores_backward(g=_tensor(_On0, 1, dtype=F32))),
    (ValueError, lambda: _scores_backward(out=_tensor(_On0, 3, 9))),
    (ValueError, lambda: _scores_backward(out=_tensor(_On0, 3, 8, dtype=F32))),
    (ValueError, lambda: _scores_backward(out=_tensor(_On0, 8, 3).t())),
    (ValueError, lambda: _scores_backward(out=_tensor(_On0, 1, 8).expand(3, 8))),
    (TypeError, lambda: _head(x=_tensor(_On0, 3, 8, dtype=F32))),
    (TypeError, lambda: _head(w=_tensor(_On0, 9, 8, dtype=F32))),
    (ValueError, lambda: _head(w=_tensor(_On0, 9, 7))),
    (ValueError, lambda: _head(w=_tensor(_On0, 72))),
    (ValueError, lambda: _head(t=_ids(_On0, 2))),
    (ValueError, lambda: _head_backward(lse=_tensor(_On0, 4, dtype=F32))),
])
def test_refusals(calls, error, call):
    with pytest.raises(error):
        call()
    assert calls == []


def test_out_that_wants_a_gradient_is_refused(calls):
    z = _tensor(_On0, 3, 8).requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        _scores_backward(z=z, out=z)
    assert calls == []


def test_rows_apart_are_taken_as_they_lie(calls):
    wide = _tensor(_On0, 2, 5, 20)
    part = wide[..., 3:11]
    gf.token_logprobs(part, _ids(_On0, 2, 5))
    name, a = calls[-1]
    assert name == "gefen_token_logprobs"
    assert a[0] == part.data_ptr() and a[1] == 20 and a[3:5] == (10, 8)
    gf.token_logprobs(wide[:1, 1:2, 3:11], _ids(_On0, 1, 1))        # one row: any distance
    assert calls[-1][1][1] == 8
    gf.token_logprobs(_tensor(_On0, 8, 6).t(), _ids(_On0, 6))       # not along its rows: a copy
    assert calls[-1][1][1] == 8
    gf.token_logprobs(_tensor(_On0, 8).expand(6, 8), _ids(_On0, 6))  # rows that overlap: a copy
    assert calls[-1][1][1] == 8
    out = _tensor(_On0, 2, 5, 30)[..., 1:9]
    f = _tensor(_On0, 2, 5, dtype=F32)
    gf.token_logprobs_backward(f, part, _ids(_On0, 2, 5), f, f, out=out)
    a = calls[-1][1]
    assert a[1] == 20 and a[11] == out.data_ptr() and a[12] == 30


def test_writing_in_place_is_seen_by_autograd(calls):
    z = _tensor(_On0, 3, 8)
    before = z._version
    assert _scores_backward(z=z, out=z) is z
    assert z._version > before


def test_seeds(calls):
    """Numbers are taken modulo 2^64; a tensor is read by the kernel."""
    gf.dropout(_tensor(_On0, 4), 0.5, -1, -2)
    a = calls[-1][1]
    assert a[5:8] == (2 ** 64 - 1, 2 ** 64 - 2, None)
    state = _ids(_On0, 2)
    gf.dropout(_tensor(_On0, 4), 0.5, state, 3)
    assert calls[-1][1][5:8] == (0, 3, state.data_ptr())


def test_unaligned_operands_ask_for_their_copies(calls, monkeypatch):
    flags = []

    def space(n, width, vocab, f, out):
        flags.append(f)
        return 0
    monkeypatch.setattr(type(ff._library()), "gefen_head_logprobs_workspace",
                        staticmethod(space), raising=False)
    buffer = torch.zeros(1 + 9 * 8, dtype=BF16)
    off = 1 if buffer.data_ptr() % 16 == 0 else 0
    w = buffer[off:off + 72].view(9, 8).as_subclass(_On0)
    assert w.data_ptr() % 16
    _head(w=w)
    _head_backward(w=w)
    assert flags == [ff._UNALIGNED, ff._UNALIGNED | ff._BACKWARD]


def test_plain_calls_carry_no_graph(calls):
    w = _tensor(_On0, 9, 8).requires_grad_()
    y = gf.embedding(_ids(_On0, 3), w)
    with pytest.raises(RuntimeError, match="Embedding has"):
        y.sum().backward()
    with torch.no_grad():
        assert not gf.embedding(_ids(_On0, 3), w).requires_grad
    z = _tensor(_On0, 3, 8).requires_grad_()
    for r, who in ((gf.dropout(z, 0.5, 1), "Dropout"), (_scores(z=z).entropy, "LogProbs"),
                   (_head(x=z).logprob, "Head"), (_head(w=w).lse, "Head")):
        with pytest.raises(RuntimeError, match=who + " has"):
            r.sum().backward()
    g = _tensor(_On0, 3, dtype=F32).requires_grad_()
    for r in (_scores_backward(g=g), *_head_backward(g=g)):
        with pytest.raises(RuntimeError, match="cannot be differentiated"):
            r.sum().backward()


def test_dropout_module():
    """Evaluation and p = 0 launch nothing and leave the numbers; p is checked."""
    for drop in (gf.Dropout(0.0), gf.Dropout(0.3).eval()):
        x, r = torch.randn(4), torch.randn(4)
        assert drop(x) is x and torch.equal(drop(x, r), x + r)
        assert drop.state.tolist() == [0, 0]
    for p in (-0.1, 1.5, math.nan):
        with pytest.raises(ValueError):
            gf.Dropout(p)
    assert gf.Dropout(0.1, seed=-5).state.tolist() == [-5, 0]
    with pytest.raises(ValueError):
        gf.FeedForward(8, 8, dropout=2.0)
    assert gf.FeedForward(8, 8).drop is None
    assert set(gf.FeedForward(8, 8).state_dict()) == {"norm", "w_gate", "w_up", "w_down"}
    assert "drop.state" in gf.FeedForward(8, 8, dropout=0.1, seed=3).state_dict()


def test_modules_share_a_table():
    emb = gf.Embedding(20, 8)
    head = gf.Head(8, 20, weight=emb.table)
    assert head.weight is emb.table
    with pytest.raises(ValueError, match="shape"):
        gf.Head(8, 21, weight=emb.table)
    assert gf.Head(8, 20).weight.shape == (20, 8)
