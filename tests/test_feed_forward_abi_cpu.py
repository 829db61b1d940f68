"""Argument errors of the feed-forward entry points, which return before touching the device."""
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


def test_checkpoint_refusals(lib):
    enc, dec = lib.gefen_checkpoint_encode, lib.gefen_checkpoint_decode
    _said(lib, enc(P, 7, 1, 1, P, P, None), -2, "dtype")
    _said(lib, enc(P, 0, -1, 1, P, P, None), -1, "rows")
    _said(lib, enc(P, 0, 1, 0, P, P, None), -1, "cols")
    _said(lib, enc(P, 0, 1 << 30, 1 << 30, P, P, None), -1, "2^40")
    _said(lib, enc(None, 0, 1, 1, P, P, None), -1, "NULL")
    _said(lib, enc(P, 0, 1, 1, P, None, None), -1, "NULL")
    _said(lib, dec(P, P, None, 1, 1, P, 2, None), -2, "dtype")
    _said(lib, dec(P, P, None, 1, 1, None, 0, None), -1, "NULL")
    assert enc(None, 0, 0, 5, None, None, None) == 0       # no rows: nothing to do


def test_norm_refusals(lib):
    def norm(x=P, r=None, dt=0, w=P, rows=2, cols=8, eps=1e-6, y=P, h=None, rstd=P, c=None, e=None):
        return lib.gefen_rms_norm(x, r, dt, w, rows, cols, eps, y, h, rstd, c, e, None)
    _said(lib, norm(dt=3), -2, "dtype")
    _said(lib, norm(cols=16385), -1, "cols")
    _said(lib, norm(rows=-1), -1, "rows")
    _said(lib, norm(eps=-1e-9), -1, "eps")
    _said(lib, norm(eps=float("inf")), -1, "eps")
    _said(lib, norm(c=P), -1, "go together")
    for name in ("x", "w", "y", "rstd"):
        _said(lib, norm(**{name: None}), -1, "NULL")
    n = ctypes.c_int64()
    assert lib.gefen_rms_norm_backward_workspace(100, 64, n) == 0 and n.value >= 4 * 64
    _said(lib, lib.gefen_rms_norm_backward_workspace(100, 64, None), -1, "NULL")

    def back(dy=P, dh=None, dt=0, h=P, c=None, e=None, rstd=P, w=P, rows=100, cols=64, dx=P, dw=P,
             ws=P, nb=1 << 30):
        return lib.gefen_rms_norm_backward(dy, dh, dt, h, c, e, rstd, w, rows, cols, dx, dw, ws,
                                           nb, None)
    _said(lib, back(h=None), -1, "either")
    _said(lib, back(c=P, e=P), -1, "either")
    _said(lib, back(h=None, c=P), -1, "either")
    _said(lib, back(nb=n.value - 1), -1, "workspace")
    _said(lib, back(ws=None), -1, "workspace")
    _said(lib, back(ws=P + 4), -1, "aligned")
    for name in ("dy", "rstd", "w", "dx", "dw"):
        _said(lib, back(**{name: None}), -1, "NULL")


def test_ffn_refusals(lib):
    n = ctypes.c_int64()
    space = lib.gefen_gated_ffn_workspace
    assert space(16, 64, 64, 0, n) == 0 and n.value >= 2 * 16 * 64
    forward = n.value
    assert space(16, 64, 64, 1, n) == 0 and n.value > forward
    backward = n.value
    assert space(16, 64, 64, 3, n) == 0 and n.value > backward
    assert space(0, 64, 64, 0, n) == 0 and n.value == 0
    _said(lib, space(16, 64, 64, 4, n), -1, "flags")
    _said(lib, space(16, 64, 64, 0, None), -1, "NULL")
    for t, k, f in ((-1, 8, 8), ((1 << 24) + 1, 8, 8), (1, 0, 8), (1, 8, 0), (1, (1 << 20) + 1, 8),
                    (1 << 24, 8, 1 << 20)):
        assert space(t, k, f, 0, n) == -1

    def fwd(x=P, wg=P, wu=P, wd=P, t=16, k=64, f=64, act=0, y=P, c=(None,) * 4, ws=P, nb=1 << 30):
        return lib.gefen_gated_ffn(x, wg, wu, wd, t, k, f, act, y, *c, ws, nb, None)
    _said(lib, fwd(act=2), -1, "activation")
    _said(lib, fwd(c=(P, P, P, None)), -1, "go together")
    _said(lib, fwd(nb=forward - 1), -1, "workspace")
    _said(lib, fwd(ws=P + 8), -1, "aligned")
    for name in ("x", "wg", "wu", "wd", "y"):
        _said(lib, fwd(**{name: None}), -1, "NULL")

    def back(dy=P, x=P, xc=None, xe=None, gain=None, c=(P,) * 4, wg=P, wu=P, wd=P, t=16, act=0,
             dx=P, dwg=P, dwu=P, dwd=P, nb=1 << 30):
        return lib.gefen_gated_ffn_backward(dy, x, xc, xe, gain, *c, wg, wu, wd, t, 64, 64, act,
                                            dx, dwg, dwu, dwd, P, nb, None)
    _said(lib, back(act=-1), -1, "activation")
    _said(lib, back(x=None), -1, "either")
    _said(lib, back(xc=P, xe=P), -1, "either")
    _said(lib, back(x=None, xc=P), -1, "either")
    _said(lib, back(gain=P), -1, "gain")
    _said(lib, back(nb=backward - 1), -1, "workspace")
    for name in ("dy", "wg", "wu", "wd", "dx", "dwg", "dwu", "dwd"):
        _said(lib, back(**{name: None}), -1, "NULL")
    _said(lib, back(c=(P, P, None, P)), -1, "NULL")
