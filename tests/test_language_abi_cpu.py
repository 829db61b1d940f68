"""Argument errors of the entry points at a language model's two ends, which return before touching
the device."""
import ctypes
import os

import pytest

P = 0x1000   # never read: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    import paper_2606_13894_amd as gf
    if not os.path.exists(gf.LIB_PATH):
        pytest.skip("libgefen.so is not built (run __graft_entry__.build())")
    return gf.load_library()


def _said(lib, rc, want, word):
    assert rc == want, lib.gefen_last_error()
    assert word.encode() in lib.gefen_last_error()


def test_embedding_refusals(lib):
    def call(t=P, tb=8, n=3, w=P, wd=0, vocab=5, width=8, scale=1.0, y=P, d=0):
        return lib.gefen_embedding(t, tb, n, w, wd, vocab, width, scale, y, d, None)
    _said(lib, call(wd=2), -2, "dtype")
    _said(lib, call(d=-1), -2, "dtype")
    _said(lib, call(tb=2), -1, "token_bytes")
    _said(lib, call(n=-1), -1, "tokens")
    _said(lib, call(n=(1 << 24) + 1), -1, "tokens")
    _said(lib, call(vocab=0), -1, "vocab")
    _said(lib, call(vocab=(1 << 24) + 1), -1, "vocab")
    _said(lib, call(width=0), -1, "width")
    _said(lib, call(width=(1 << 20) + 1), -1, "width")
    _said(lib, call(vocab=1 << 24, width=1 << 20), -1, "2^40")
    _said(lib, call(n=1 << 24, width=1 << 20), -1, "2^40")
    for s in (float("nan"), float("inf"), 1e39):
        _said(lib, call(scale=s), -1, "scale")
    for name in ("t", "w", "y"):
        _said(lib, call(**{name: None}), -1, "NULL")
    assert call(t=None, w=None, y=None, n=0) == 0


def test_embedding_backward_refusals(lib):
    n = ctypes.c_int64()
    space = lib.gefen_embedding_backward_workspace
    assert space(100, 50, 64, n) == 0 and n.value >= 4 * 4 * 100
    _said(lib, space(100, 50, 64, None), -1, "NULL")
    _said(lib, space(-1, 50, 64, n), -1, "tokens")
    _said(lib, space(100, 0, 64, n), -1, "vocab")
    assert space(100, 50, 64, n) == 0

    def call(dy=P, d=0, t=P, tb=8, rows=100, vocab=50, width=64, scale=1.0, g=P, gd=0, ws=P,
             nb=n.value):
        return lib.gefen_embedding_backward(dy, d, t, tb, rows, vocab, width, scale, g, gd, ws, nb,
                                            None)
    _said(lib, call(d=9), -2, "dtype")
    _said(lib, call(gd=9), -2, "dtype")
    _said(lib, call(tb=1), -1, "token_bytes")
    _said(lib, call(scale=float("inf")), -1, "scale")
    _said(lib, call(nb=n.value - 1), -1, "workspace")
    _said(lib, call(ws=None), -1, "workspace")
    _said(lib, call(ws=P + 8), -1, "aligned")
    for name in ("dy", "t", "g"):
        _said(lib, call(**{name: None}), -1, "NULL")


def test_dropout_refusals(lib):
    def call(x=P, r=None, d=1, n=8, p=0.1, y=P):
        return lib.gefen_dropout(x, r, d, n, p, 1, 0, None, y, None)
    _said(lib, call(d=4), -2, "dtype")
    _said(lib, call(n=-1), -1, "n must be")
    _said(lib, call(n=(1 << 40) + 1), -1, "n must be")
    for p in (-0.1, 1.1, float("nan")):
        _said(lib, call(p=p), -1, "p must be")
    _said(lib, call(x=None), -1, "NULL")
    _said(lib, call(y=None), -1, "NULL")
    assert call(x=None, y=None, n=0) == 0


def test_token_logprobs_refusals(lib):
    n = ctypes.c_int64()
    space = lib.gefen_token_logprobs_workspace
    _said(lib, space(5, 1, 10, 0, n), -2, "dtype")
    _said(lib, space(0, -1, 10, 0, n), -1, "rows")
    _said(lib, space(0, 1, 0, 0, n), -1, "vocab")
    _said(lib, space(0, 1, 10, 11, n), -1, "top")
    _said(lib, space(0, 1, 100, 33, n), -1, "top")
    _said(lib, space(0, 1, 100, 5, None), -1, "NULL")
    assert space(0, 1, 1_000_000, 5, n) == 0 and n.value > 0

    def call(z=P, ld=1_000_000, d=0, rows=1, vocab=1_000_000, t=P, tb=8, top=5, lp=P, e=P, l=P, b=P,
             w=P, ws=P, nb=n.value):
        return lib.gefen_token_logprobs(z, ld, d, rows, vocab, t, tb, top, lp, e, l, b, w, ws, nb,
                                        None)
    _said(lib, call(d=3), -2, "dtype")
    _said(lib, call(ld=999_999), -1, "overlap")
    _said(lib, call(rows=1 << 30), -1, "2^40")
    _said(lib, call(tb=3), -1, "token_bytes")
    _said(lib, call(top=-1), -1, "top")
    _said(lib, call(nb=n.value - 1), -1, "workspace")
    _said(lib, call(ws=P + 4), -1, "aligned")
    for name in ("z", "t", "lp", "e", "l", "b", "w"):
        _said(lib, call(**{name: None}), -1, "NULL")
    assert call(rows=0, z=None) == 0

    def back(z=P, ld=100, d=0, rows=2, vocab=100, t=P, tb=8, l=P, e=P, g=P, h=None, o=P, ldd=100):
        return lib.gefen_token_logprobs_backward(z, ld, d, rows, vocab, t, tb, l, e, g, h, o, ldd,
                                                 None)
    _said(lib, back(d=3), -2, "dtype")
    _said(lib, back(ld=99), -1, "overlap")
    _said(lib, back(ldd=99), -1, "overlap")
    _said(lib, back(ldd=120), -1, "as far apart")
    _said(lib, back(tb=16), -1, "token_bytes")
    for name in ("z", "t", "l", "e", "g", "o"):
        _said(lib, back(**{name: None}), -1, "NULL")


def test_head_refusals(lib):
    n = ctypes.c_int64()
    space = lib.gefen_head_logprobs_workspace
    _said(lib, space(10, 64, 100, 4, n), -1, "flags")
    _said(lib, space(10, 64, 100, 0, None), -1, "NULL")
    _said(lib, space(-1, 64, 100, 0, n), -1, "tokens")
    _said(lib, space(10, 0, 100, 0, n), -1, "width")
    _said(lib, space(10, 64, 0, 0, n), -1, "vocab")
    _said(lib, space(1 << 24, 64, 1 << 20, 0, n), -1, "2^40")
    assert space(10, 64, 100, 1, n) == 0
    back_bytes = n.value
    assert space(10, 64, 100, 0, n) == 0

    def call(x=P, w=P, t=P, tb=8, rows=10, width=64, vocab=100, lp=P, e=P, l=P, ws=P, nb=n.value):
        return lib.gefen_head_logprobs(x, w, t, tb, rows, width, vocab, lp, e, l, ws, nb, None)
    _said(lib, call(tb=0), -1, "token_bytes")
    _said(lib, call(nb=n.value - 1), -1, "workspace")
    _said(lib, call(ws=None), -1, "workspace")
    _said(lib, call(ws=P + 2), -1, "aligned")
    for name in ("x", "w", "t", "lp", "e", "l"):
        _said(lib, call(**{name: None}), -1, "NULL")
    assert call(rows=0, x=None) == 0

    def back(x=P, w=P, t=P, tb=8, rows=10, width=64, vocab=100, l=P, e=P, g=P, h=None, dx=P, dw=P,
             ws=P, nb=back_bytes):
        return lib.gefen_head_logprobs_backward(x, w, t, tb, rows, width, vocab, l, e, g, h, dx, dw,
                                                ws, nb, None)
    _said(lib, back(tb=0), -1, "token_bytes")
    _said(lib, back(nb=back_bytes - 1), -1, "workspace")
    for name in ("x", "w", "t", "l", "e", "g"):
        _said(lib, back(**{name: None}), -1, "NULL")
    _said(lib, back(dx=None, dw=None), -1, "NULL")
    assert back(rows=0, x=None, dx=None, dw=None) == 0
