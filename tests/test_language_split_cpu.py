"""The entries that keep lse in two numbers: their argument errors, and which of them the module takes."""
import ctypes

from test_language_abi_cpu import P, _said, lib  # noqa: F401
from test_language_calls_cpu import F32, _ids, _On0, _tensor, calls  # noqa: F401

import paper_2606_13894_amd as gf


def test_refusals(lib):  # noqa: F811
    n = ctypes.c_int64()
    assert lib.gefen_token_logprobs_workspace(0, 1, 1_000_000, 5, n) == 0

    def call(z=P, ld=1_000_000, d=0, rows=1, vocab=1_000_000, t=P, tb=8, top=5, lp=P, e=P, l=P, x=P,
             b=P, w=P, ws=P, nb=n.value):
        return lib.gefen_token_logprobs_split(z, ld, d, rows, vocab, t, tb, top, lp, e, l, x, b, w,
                                              ws, nb, None)
    _said(lib, call(d=3), -2, "dtype")
    _said(lib, call(ld=999_999), -1, "overlap")
    _said(lib, call(nb=n.value - 1), -1, "workspace")
    for name in ("z", "t", "lp", "e", "l", "x", "b", "w"):
        _said(lib, call(**{name: None}), -1, "NULL")
    assert call(rows=0, z=None, x=None) == 0

    def back(z=P, ld=100, d=0, rows=2, vocab=100, t=P, tb=8, l=P, x=P, e=P, g=P, h=None, o=P, ldd=100):
        return lib.gefen_token_logprobs_backward_split(z, ld, d, rows, vocab, t, tb, l, x, e, g, h, o,
                                                       ldd, None)
    _said(lib, back(d=3), -2, "dtype")
    _said(lib, back(ldd=99), -1, "overlap")
    for name in ("z", "t", "l", "x", "e", "g", "o"):
        _said(lib, back(**{name: None}), -1, "NULL")
    assert back(rows=0, z=None, x=None) == 0


def test_who_takes_them(calls):  # noqa: F811
    """The module, and its backward pass with the number that the forward pass wrote; the plain calls take
    the plain ones."""
    from paper_2606_13894_amd import language as lm
    z, t, f32 = _tensor(_On0, 3, 8), _ids(_On0, 3), _tensor(_On0, 3, dtype=F32)
    gf.LogProbs()(z, t)
    rest = _tensor(_On0, 3, dtype=F32)
    lm._token_logprobs_backward(f32, z, t, f32, rest, f32, None, None)
    gf.token_logprobs(z, t)
    gf.token_logprobs_backward(f32, z, t, f32, f32)
    assert [n for n, _ in calls] == [
        "gefen_token_logprobs_split", "gefen_token_logprobs_backward_split", "gefen_token_logprobs",
        "gefen_token_logprobs_backward"]
    lse, other = calls[0][1][10:12]
    assert lse and other and lse != other
    assert calls[1][1][7:10] == (f32.data_ptr(), rest.data_ptr(), f32.data_ptr())
