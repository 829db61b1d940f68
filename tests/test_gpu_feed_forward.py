"""The feed-forward operators (8-bit checkpoints, RMS norm, gated block) on the device against
float64 formulas.

Bounds. Rounding to bfloat16 moves a value by at most 2^-8 of it; a float32 sum of n terms is off
by at most n 2^-24 of the sum of their magnitudes. Matrix products of rounded matrices are
bounded by those two, term by term: with A rounded, |error of A W| <= 2^-8 |A| |W| + (n 2^-24) |A|
|W|, and 2^-8 of the result for the output's own rounding. float32 functions (exp, division,
square root) are taken as 16 units in the last place, 2^-20."""
import ctypes
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
ROUND = 2.0 ** -8
FLOAT = 2.0 ** -20
DTYPES = {"bf16": BF16, "f32": F32}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    return torch.device("cuda", 0)


def _randn(dev, *shape, seed=0, dtype=F32):
    gen = torch.Generator(device=dev).manual_seed(seed)
    return torch.randn(*shape, generator=gen, device=dev).to(dtype)


def _within(got, want, bound, what):
    got, want = got.to(F64), want.to(F64)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    over = (got - want).abs() - bound
    over = over[~torch.isnan(over)]
    assert over.numel() == 0 or over.max().item() <= 0.0, (what, over.max().item())


# ------------------------------------------------------------------ 8-bit checkpoints
def _groups(x):
    """x (float64 rows) in groups of 64, the last one padded with zeros."""
    rows, cols = x.shape
    n = -(-cols // 64)
    return torch.nn.functional.pad(x, (0, 64 * n - cols)).view(rows, n, 64)


def _encode64(x):
    """Codes and exponents by the definition, searched upward from the smallest exponent."""
    g = _groups(x.to(F64))
    top = g.abs().amax(2)
    bad = ~torch.isfinite(g).all(2)
    e = torch.ones_like(top, dtype=torch.int64)
    for k in range(2, 249):
        step = 2.0 ** (k - 1 - 127)
        e = torch.where((top / step).round() > 127, torch.full_like(e, k), e)
    e = torch.where(bad, torch.full_like(e, 255), e)
    step = torch.pow(torch.full_like(top, 2.0), (e - 127).to(F64))
    codes = torch.where(bad[:, :, None], torch.zeros_like(g), (g / step[:, :, None]).round())
    codes = codes.clamp(-127, 127)
    return codes.reshape(x.shape[0], -1)[:, :x.shape[1]].to(torch.int8), e.to(torch.uint8)


def _decode64(c):
    e = c.exponents.to(F64).repeat_interleave(64, -1)[..., :c.codes.shape[-1]]
    v = c.codes.to(F64) * torch.exp2(e - 127)
    return torch.where(e == 255, torch.full_like(v, math.nan), v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 63), (5, 64), (2, 65), (7, 130), (1, 2048),
                                       (33, 1601), (300, 8), (70, 512), (2, 20000)])
def test_checkpoint_codes(dev, rows, cols, dtype):
    scale = torch.exp(4 * _randn(dev, 1, cols, seed=1))
    x = (_randn(dev, rows, cols, seed=2) * scale).to(DTYPES[dtype])
    c = gf.checkpoint8(x)
    codes, exps = _encode64(x.cpu())
    assert torch.equal(c.codes.cpu(), codes)
    assert torch.equal(c.exponents.cpu(), exps)
    for out in (BF16, F32):
        y = c.decode(out)
        assert y.dtype is out
        assert torch.equal(y.cpu().to(F64), _decode64(gf.Checkpoint8(c.codes, c.exponents)).cpu())
    # the error is at most half a step, a step at most 1 / 63.5 of the group's largest
    top = _groups(x.to(F64)).abs().amax(2).repeat_interleave(64, 1)[:, :cols]
    _within(c.decode(F32), x, 0.5 * top / 63.5, "half a step")


def test_checkpoint_extremes(dev):
    tiny, big = 2.0 ** -149, torch.finfo(F32).max
    rows = [[0.0] * 4, [tiny, -3 * tiny, 0, 0], [2.0 ** -126, 2.0 ** -121, 0, 0], [big, -big, 1, 0],
            [127.5, 1.5, 0, 0], [127.49, -0.5, 2.5, 3.5], [-128.0, 127, 1, 1], [63.75, 1, 0, 0],
            [math.inf, 1, 2, 3], [1, -math.inf, 2, 3], [math.nan, 1, 2, 3], [-0.0, 0, 0, 0]]
    x = torch.tensor(rows, dtype=F32).repeat_interleave(20, 1)
    c = gf.checkpoint8(x.to(dev))
    codes, exps = _encode64(x)
    assert torch.equal(c.codes.cpu(), codes) and torch.equal(c.exponents.cpu(), exps)
    y = c.decode(F32).cpu()
    assert torch.isnan(y[8:11]).all(dim=1).tolist() == [False] * 3   # the second group is finite
    assert torch.isnan(y[8:11, :64]).all()
    assert torch.isfinite(y[:8]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_checkpoint_gain_alignment_and_views(dev, dtype):
    dt = DTYPES[dtype]
    flat = _randn(dev, 5 * 130 + 1, seed=3).to(dt)
    x = flat[1:].view(5, 130)                       # off by one element
    c = gf.checkpoint8(x)
    assert torch.equal(c.codes, gf.checkpoint8(x.clone()).codes)
    t = _randn(dev, 130, 6, seed=4).to(dt).t()      # transposed
    assert torch.equal(gf.checkpoint8(t).codes, gf.checkpoint8(t.contiguous()).codes)
    gain = _randn(dev, 130, seed=5)
    want = _decode64(c) * gain.to(F64)
    _within(c.decode(F32, gain=gain), want, 2.0 ** -23 * want.abs(), "gain")
    out = torch.empty(5 * 130 + 1, dtype=dt, device=dev)[1:].view(5, 130)
    assert c.decode(out=out) is out
    assert torch.equal(out.to(F64), _decode64(c))


# ------------------------------------------------------------------ RMS norm
WIDTHS = [1, 7, 64, 100, 512, 513, 768, 1024, 1601, 2048, 2050, 4096, 5000, 8192, 8193, 16384]


def _norm64(x, r, w, eps):
    h = x.to(F64) + (r.to(F64) if r is not None else 0.0)
    rstd = (h.pow(2).mean(-1) + eps) ** -0.5
    n = h * rstd[..., None]
    return h, rstd, n, n * w.to(F64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_forward(dev, cols, dtype):
    dt = DTYPES[dtype]
    rounding = ROUND if dt is BF16 else 2.0 ** -24
    sums = 2.0 ** -24 * (cols / 64 + 64) + FLOAT
    for rows, res in ((1, True), (5, False), (70, True)):
        x = _randn(dev, rows, cols, seed=1).to(dt)
        r = _randn(dev, rows, cols, seed=2).to(dt) if res else None
        w = 1 + 0.3 * _randn(dev, cols, seed=3)
        out = gf.rms_norm(x, w, residual=r, eps=1e-5, checkpoint=True)
        h, rstd, n, y = _norm64(x, r, w, 1e-5)
        _within(out.rstd, rstd, sums * rstd, "rstd")
        _within(out.y, y, (rounding + 2 * sums) * y.abs(), "y")
        if res:
            _within(out.h, h, rounding * h.abs(), "h")
        else:
            assert out.h is x
        step = torch.exp2(out.checkpoint.exponents.to(F64) - 127).repeat_interleave(64, 1)[:, :cols]
        _within(_decode64(out.checkpoint), n, 0.5 * step + 2 * sums * n.abs(), "saved")
        top = _groups(n).abs().amax(2)
        step = torch.exp2(out.checkpoint.exponents.to(F64) - 127)
        least = out.checkpoint.exponents == 1       # a group of zeros (x + residual = 0)
        assert (top / step <= 127.5 * 1.0001).all()
        assert ((top / step >= 63.75 * 0.9999) | least).all()
        plain = gf.rms_norm(x, w, residual=r, eps=1e-5)
        assert plain.checkpoint is None and torch.equal(plain.y, out.y)


def _norm_grad64(dy, n, rstd, w, dh):
    dy, w, rstd = dy.to(F64), w.to(F64), rstd.to(F64)[:, None]
    dn = dy * w
    c = (dn * n).mean(1, keepdim=True)
    dx = rstd * (dn - n * c)
    scale = rstd * (dn.abs() + n.abs() * (dn * n).abs().mean(1, keepdim=True))
    if dh is not None:
        dx, scale = dx + dh.to(F64), scale + dh.to(F64).abs()
    return dx, (dy * n).sum(0), scale, (dy * n).abs().sum(0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("saved", ["codes", "h"])
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_backward(dev, cols, saved, dtype):
    dt = DTYPES[dtype]
    rounding = ROUND if dt is BF16 else 2.0 ** -24
    for rows, res in ((1, False), (6, True), (1300, True)):
        x = _randn(dev, rows, cols, seed=4).to(dt)
        w = 1 + 0.3 * _randn(dev, cols, seed=5)
        dy = _randn(dev, rows, cols, seed=6).to(dt)
        dh = _randn(dev, rows, cols, seed=7).to(dt) if res else None
        out = gf.rms_norm(x, w, checkpoint=True)
        keep = out.checkpoint if saved == "codes" else out.h
        n = _decode64(out.checkpoint) if saved == "codes" else \
            x.to(F64) * out.rstd.to(F64)[:, None]
        dx, dw = gf.rms_norm_backward(dy, keep, out.rstd, w, dh=dh)
        want, want_w, scale, scale_w = _norm_grad64(dy, n, out.rstd, w, dh)
        sums = 2.0 ** -24 * (cols / 64 + 64) + FLOAT
        _within(dx, want, sums * scale + rounding * want.abs(), "dx")
        _within(dw, want_w, 2.0 ** -24 * (rows + 8) * scale_w, "dweight")
        again = gf.rms_norm_backward(dy, keep, out.rstd, w, dh=dh)
        assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


def test_norm_gradient_by_differences(dev):
    rows, cols, eps = 4, 37, 1e-4
    x, r = _randn(dev, rows, cols, seed=8), _randn(dev, rows, cols, seed=9)
    w = 1 + 0.3 * _randn(dev, cols, seed=10)
    dy, dh = _randn(dev, rows, cols, seed=11), _randn(dev, rows, cols, seed=12)
    out = gf.rms_norm(x, w, residual=r, eps=1e-5)
    dx, dw = gf.rms_norm_backward(dy, out.h, out.rstd, w, dh=dh)

    def loss(a, b, c):
        h, _, _, y = _norm64(a, b, c, 1e-5)
        return ((y * dy.to(F64)).sum() + (h * dh.to(F64)).sum()).item()

    for k in range(5):
        a = _randn(dev, rows, cols, seed=20 + k).to(F64)
        c = _randn(dev, cols, seed=30 + k).to(F64)
        xs, rs, ws = x.to(F64), r.to(F64), w.to(F64)
        for move, got in (((a, 0, 0), (dx.to(F64) * a).sum()), ((0, a, 0), (dx.to(F64) * a).sum()),
                          ((0, 0, c), (dw.to(F64) * c).sum())):
            up = loss(xs + eps * move[0], rs + eps * move[1], ws + eps * move[2])
            down = loss(xs - eps * move[0], rs - eps * move[1], ws - eps * move[2])
            # float32 gradients of a few hundred terms of size 1; the differences' own error is
            # eps^2 times the third derivative
            assert abs((up - down) / (2 * eps) - got.item()) < 2e-4


def test_norm_edges(dev):
    w = torch.ones(100, device=dev)
    z = torch.zeros(3, 100, device=dev)
    out = gf.rms_norm(z, w, eps=1e-6, checkpoint=True)
    assert not out.y.any() and not out.checkpoint.codes.any()
    assert torch.allclose(out.rstd, torch.full_like(out.rstd, 1e3))
    x = _randn(dev, 4, 100, seed=1)
    clean = gf.rms_norm(x, w, checkpoint=True)
    x[2, 17] = math.nan
    out = gf.rms_norm(x, w, checkpoint=True)
    assert torch.isnan(out.y[2]).all() and torch.isnan(out.checkpoint.decode()[2]).all()
    keep = [0, 1, 3]
    assert torch.equal(out.y[keep], clean.y[keep])
    assert torch.equal(out.checkpoint.codes[keep], clean.checkpoint.codes[keep])
    dx, dw = gf.rms_norm_backward(x * 0 + 1, out.checkpoint, out.rstd, w)
    assert torch.isnan(dx[2]).all() and not torch.isnan(dx[keep]).any() and torch.isnan(dw).all()
    e = torch.empty(0, 100, device=dev)
    out = gf.rms_norm(e, w, checkpoint=True)
    assert out.y.shape == (0, 100)
    dx, dw = gf.rms_norm_backward(e, out.checkpoint, out.rstd, w)
    assert dx.shape == (0, 100) and not dw.any()
    x3 = _randn(dev, 2, 3, 100, seed=2)             # leading dimensions, a transposed view
    assert torch.equal(gf.rms_norm(x3, w).y.view(6, 100), gf.rms_norm(x3.view(6, 100), w).y)
    t = _randn(dev, 100, 6, seed=3).t()
    assert torch.equal(gf.rms_norm(t, w).y, gf.rms_norm(t.contiguous(), w).y)
    off = _randn(dev, 3 * 101 + 1, seed=4).to(BF16)[1:].view(3, 101)
    w1 = torch.ones(102, device=dev)[1:]
    assert torch.equal(gf.rms_norm(off, w1).y, gf.rms_norm(off.clone(), w1.clone()).y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [5, 100, 777, 1601, 2048, 4099, 8191, 8201, 8205, 12289, 16384])
def test_norm_in_place(dev, cols, dtype):
    """y and h may be x or the residual, dx may be dy or dh: the same bits either way."""
    lib, p = gf.load_library(), lambda t: None if t is None else t.data_ptr()
    rows, dt = 1000 if cols < 4000 else 300, {"bf16": BF16, "f32": F32}[dtype]
    d = gf.BF16 if dt is BF16 else gf.F32
    stream = torch.cuda.current_stream().cuda_stream
    x, r, dy, dh = (_randn(dev, rows, cols, seed=i, dtype=dt) for i in range(4))
    w = 1 + 0.1 * _randn(dev, cols, seed=5)
    rstd = torch.empty(rows, device=dev)

    def forward(a, b, y, h):
        assert lib.gefen_rms_norm(p(a), p(b), d, p(w), rows, cols, 1e-6, p(y), p(h), p(rstd), None,
                                  None, stream) == 0
        return y, h

    y, h = forward(x, r, torch.empty_like(x), torch.empty_like(x))
    for swap in (False, True):
        a, b = x.clone(), r.clone()
        got = forward(a, b, b, a) if swap else forward(a, b, a, b)
        assert torch.equal(got[0], y) and torch.equal(got[1], h)

    n = ctypes.c_int64()
    assert lib.gefen_rms_norm_backward_workspace(rows, cols, ctypes.byref(n)) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device=dev)
    code = gf.checkpoint8(h.float() * rstd[:, None])

    def backward(a, b, dx, saved):
        dw = torch.empty(cols, device=dev)
        of = (p(h), None, None) if saved == "h" else (None, p(code.codes), p(code.exponents))
        assert lib.gefen_rms_norm_backward(p(a), p(b), d, *of, p(rstd), p(w), rows, cols, p(dx),
                                           p(dw), p(ws), n.value, stream) == 0
        return dx, dw

    for saved in ("h", "codes"):
        want = backward(dy, dh, torch.empty_like(dy), saved)
        a, b = dy.clone(), dh.clone()
        for got in (backward(a, dh, a, saved), backward(dy, b, b, saved)):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ------------------------------------------------------------------ the gated block
def _act64(g, act):
    z = g if act == "silu" else 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    return g * torch.sigmoid(z)


def _slope64(g, act):
    g = g.clone().requires_grad_(True)
    (s,) = torch.autograd.grad(_act64(g, act).sum(), g)
    return s


def _ffn_inputs(dev, T, K, F, seed=0):
    x = _randn(dev, T, K, seed=seed + 1).to(BF16)
    wg = (_randn(dev, F, K, seed=seed + 2) * K ** -0.5).to(BF16)
    wu = (_randn(dev, F, K, seed=seed + 3) * K ** -0.5).to(BF16)
    wd = (_randn(dev, K, F, seed=seed + 4) * F ** -0.5).to(BF16)
    dy = _randn(dev, T, K, seed=seed + 5).to(BF16)
    return x, wg, wu, wd, dy


def _check_forward(x, wg, wu, wd, act, y, saved):
    T, K = x.shape
    F = wg.shape[0]
    xd, gd, ud, dd = (t.to(F64) for t in (x, wg, wu, wd))
    g, u = xd @ gd.t(), xd @ ud.t()
    g_err = (K * 2.0 ** -24) * (xd.abs() @ gd.abs().t())
    u_err = (K * 2.0 ** -24) * (xd.abs() @ ud.abs().t())
    a = _act64(g, act) * u
    # |act'| <= 1.13, |act| <= |g|
    a_err = 1.2 * g_err * u.abs() + g.abs() * u_err + 2 * FLOAT * (g * u).abs() + ROUND * a.abs()
    want = a @ dd.t()
    _within(y, want, ROUND * want.abs() * 1.01 + a_err @ dd.abs().t()
            + F * 2.0 ** -24 * (a.abs() @ dd.abs().t()), "y")
    if saved is None:
        return
    for c, v, err in ((saved[0], g, g_err), (saved[1], u, u_err)):
        step = torch.exp2(c.exponents.to(F64) - 127)
        wide = step.repeat_interleave(64, 1)[:, :F]
        _within(_decode64(c), v, 0.5 * wide + err, "saved")
        top = _groups(v).abs().amax(2)
        slack = _groups(err).amax(2)
        assert ((top - slack) / step <= 127.5).all()
        assert ((top + slack) / step >= 63.75).all()


def _check_backward(dy, xs, saved, wg, wu, wd, act, grads, gain=None):
    """xs: float64 input of the weight gradients, without its gain."""
    T, K = dy.shape
    F = wg.shape[0]
    dd, gd, ud, yd = (t.to(F64) for t in (wd, wg, wu, dy))
    g, u = _decode64(saved[0]), _decode64(saved[1])
    da = yd @ dd
    da_err = K * 2.0 ** -24 * (yd.abs() @ dd.abs())
    av, slope = _act64(g, act), _slope64(g, act)
    dg, du, a = da * u * slope, da * av, av * u
    # float32 activation: FLOAT of its terms' sizes (|slope| <= 1.2, |act| <= |g|)
    dg_err = 1.2 * da_err * u.abs() + 4 * FLOAT * (da * u).abs() * (1 + g.abs()) + ROUND * dg.abs()
    du_err = da_err * av.abs() + 2 * FLOAT * (da * g).abs() + ROUND * du.abs()
    a_err = 2 * FLOAT * (g * u).abs() + ROUND * a.abs()
    dx, dwg, dwu, dwd = grads
    want = dg @ gd + du @ ud
    size = dg.abs() @ gd.abs() + du.abs() @ ud.abs()
    _within(dx, want, ROUND * want.abs() * 1.02 + dg_err @ gd.abs() + du_err @ ud.abs()
            + 2 * F * 2.0 ** -24 * size, "dx")
    col = 1.0 if gain is None else gain.to(F64).abs()
    sgn = 1.0 if gain is None else gain.to(F64)
    for got, d, err, what in ((dwg, dg, dg_err, "dw_gate"), (dwu, du, du_err, "dw_up")):
        want = (d.t() @ xs) * sgn
        _within(got, want, ROUND * want.abs() * 1.02 + (err.t() @ xs.abs()) * col
                + T * 2.0 ** -24 * (d.abs().t() @ xs.abs()) * col, what)
    want = yd.t() @ a
    _within(dwd, want, ROUND * want.abs() * 1.02 + yd.abs().t() @ a_err
            + T * 2.0 ** -24 * (yd.abs().t() @ a.abs()), "dw_down")


SIZES = [(1, 64, 64), (1, 2048, 512), (2, 8, 8), (3, 1, 1), (5, 9, 7), (16, 256, 130),
         (17, 100, 63), (33, 72, 40), (48, 136, 65), (64, 512, 256), (65, 130, 190),
         (128, 128, 128), (129, 264, 200), (200, 320, 72), (256, 256, 256), (300, 765, 515),
         (257, 520, 24), (1000, 64, 300), (777, 96, 1040)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,K,F", SIZES)
def test_ffn(dev, T, K, F, act):
    x, wg, wu, wd, dy = _ffn_inputs(dev, T, K, F, seed=T)
    y, saved = gf.gated_ffn(x, wg, wu, wd, activation=act, checkpoint=True)
    _check_forward(x, wg, wu, wd, act, y, saved)
    plain = gf.gated_ffn(x, wg, wu, wd, activation=act)
    _check_forward(x, wg, wu, wd, act, plain, None)
    grads = gf.gated_ffn_backward(dy, x, saved, wg, wu, wd, activation=act)
    _check_backward(dy, x.to(F64), saved, wg, wu, wd, act, grads)
    again = gf.gated_ffn_backward(dy, x, saved, wg, wu, wd, activation=act)
    assert all(torch.equal(p, q) for p, q in zip(grads, again))
    gain = 1 + 0.3 * _randn(dev, K, seed=99)
    xc = gf.checkpoint8(x)
    grads = gf.gated_ffn_backward(dy, xc, saved, wg, wu, wd, activation=act, gain=gain)
    _check_backward(dy, _decode64(xc), saved, wg, wu, wd, act, grads, gain)


@pytest.mark.parametrize("T,K,F", [(700, 512, 2048), (2048, 512, 256), (600, 1536, 640),
                                   (4100, 260, 1030), (24, 4096, 1024)])
def test_ffn_larger(dev, T, K, F):
    """Sizes whose products take the larger tile, or split sums."""
    test_ffn(dev, T, K, F, "silu")


def test_ffn_alignment_and_views(dev):
    T, K, F = 40, 72, 136
    x, wg, wu, wd, dy = _ffn_inputs(dev, T, K, F)
    y, saved = gf.gated_ffn(x, wg, wu, wd, checkpoint=True)
    grads = gf.gated_ffn_backward(dy, x, saved, wg, wu, wd)

    def off(t):   # the same values, two bytes past an aligned address
        s = torch.empty(t.numel() + 1, dtype=t.dtype, device=dev)[1:].view(t.shape)
        s.copy_(t)
        return s

    for i in range(4):
        ops = [x, wg, wu, wd]
        ops[i] = off(ops[i])
        y2, s2 = gf.gated_ffn(*ops, checkpoint=True)
        assert torch.equal(y, y2) and torch.equal(saved[0].codes, s2[0].codes)
        got = gf.gated_ffn_backward(dy, ops[0], saved, *ops[1:])
        assert all(torch.equal(p, q) for p, q in zip(grads, got))
    got = gf.gated_ffn_backward(off(dy), x, saved, wg, wu, wd)
    assert all(torch.equal(p, q) for p, q in zip(grads, got))
    wt = wg.t().contiguous().t()                    # column-major weights
    assert torch.equal(y, gf.gated_ffn(x, wt, wu, wd, checkpoint=True)[0])
    y3, s3 = gf.gated_ffn(x.view(5, 8, K), wg, wu, wd, checkpoint=True)
    assert torch.equal(y3.view(T, K), y) and s3[0].shape == (5, 8, F)
    g3 = gf.gated_ffn_backward(dy.view(5, 8, K), x.view(5, 8, K), s3, wg, wu, wd)
    assert torch.equal(g3[0].view(T, K), grads[0]) and torch.equal(g3[3], grads[3])


def test_ffn_gradient_by_differences(dev):
    """Directional differences of the float64 block against the gradients from 8-bit checkpoints
    (rounding noise of a hundredth of each factor, averaged over thousands of terms)."""
    T, K, F, eps = 24, 64, 96, 1e-4
    x, wg, wu, wd, dy = _ffn_inputs(dev, T, K, F, seed=50)
    _, saved = gf.gated_ffn(x, wg, wu, wd, "gelu", checkpoint=True)
    grads = [g.to(F64) for g in gf.gated_ffn_backward(dy, x, saved, wg, wu, wd, "gelu")]
    base = [t.to(F64) for t in (x, wg, wu, wd)]

    def loss(p):
        return (((_act64(p[0] @ p[1].t(), "gelu") * (p[0] @ p[2].t())) @ p[3].t())
                * dy.to(F64)).sum().item()

    for i in range(4):
        for k in range(4):
            d = _randn(dev, *base[i].shape, seed=60 + k).to(F64)
            up = [b + eps * d if j == i else b for j, b in enumerate(base)]
            down = [b - eps * d if j == i else b for j, b in enumerate(base)]
            want = (loss(up) - loss(down)) / (2 * eps)
            got = (grads[i] * d).sum().item()
            assert abs(want - got) <= 0.05 * grads[i].norm().item(), (i, k)


def test_ffn_edges(dev):
    T, K, F = 70, 136, 72
    x, wg, wu, wd, dy = _ffn_inputs(dev, T, K, F)
    y, saved = gf.gated_ffn(x, wg, wu, wd, checkpoint=True)
    clean = gf.gated_ffn_backward(dy, x, saved, wg, wu, wd)
    bad = x.clone()
    bad[33, 5] = math.nan
    yb, sb = gf.gated_ffn(bad, wg, wu, wd, checkpoint=True)
    keep = [t for t in range(T) if t != 33]
    assert torch.isnan(yb[33]).all() and torch.equal(yb[keep], y[keep])
    assert torch.equal(sb[0].codes[keep], saved[0].codes[keep])
    dx, dwg, _, dwd = gf.gated_ffn_backward(dy, bad, sb, wg, wu, wd)
    assert torch.isnan(dx[33]).all() and torch.equal(dx[keep], clean[0][keep])
    assert torch.isnan(dwg).all() and torch.isnan(dwd).all()
    zero = gf.gated_ffn(torch.zeros_like(x), wg, wu, wd, checkpoint=True)
    assert not zero[0].any() and not zero[1][0].codes.any()
    e = torch.empty(0, K, dtype=BF16, device=dev)
    ye, se = gf.gated_ffn(e, wg, wu, wd, checkpoint=True)
    assert ye.shape == (0, K)
    ge = gf.gated_ffn_backward(e, e, se, wg, wu, wd)
    assert ge[0].shape == (0, K) and not any(g.any() for g in ge[1:])
    # large gates: the logistic saturates without NaN
    big = gf.gated_ffn((x.float() * 1000).to(BF16), wg, wu, wd, "gelu", checkpoint=True)
    assert torch.isfinite(big[0]).all()
    gb = gf.gated_ffn_backward(dy, x, big[1], wg, wu, wd, "gelu")
    assert all(torch.isfinite(g).all() for g in gb)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_ffn_huge_gates(dev, act):
    """Gates whose square passes float32: the activation is the gate or zero, its slope one or
    zero, as the formulas' limits are."""
    T, K, F = 40, 64, 96
    x, wg, wu, wd, dy = _ffn_inputs(dev, T, K, F, seed=7)
    wg, wd = (wg.float() * 2.0 ** 70).to(BF16), (wd.float() * 2.0 ** -70).to(BF16)
    y, saved = gf.gated_ffn(x, wg, wu, wd, act, checkpoint=True)
    assert torch.isfinite(y).all()
    grads = gf.gated_ffn_backward(dy, x, saved, wg, wu, wd, act)
    assert all(torch.isfinite(g).all() for g in grads)
    g, u = _decode64(saved[0]), _decode64(saved[1])
    big = g.abs() > 2.0 ** 40            # all but the codes 0
    on = (big & (g > 0)).to(F64)
    da = dy.to(F64) @ wd.to(F64)
    keep = big | (g == 0)
    assert keep.all()
    slope = torch.where(g == 0, torch.full_like(g, 0.5), on)
    dg = da * u * slope
    want = dg.t() @ x.to(F64)
    _within(grads[1], want, ROUND * want.abs() * 1.02 + (2 * ROUND * dg.abs()).t() @ x.to(F64).abs(),
            "dw_gate")
    a = torch.where(g > 0, g, torch.zeros_like(g)) * u
    want = dy.to(F64).t() @ a
    _within(grads[3], want, ROUND * want.abs() * 1.02 + dy.to(F64).abs().t() @ (2 * ROUND * a.abs()),
            "dw_down")


def test_ffn_infinity_stays_infinity(dev):
    """An infinite input and positive weights: infinite outputs, whatever is padded."""
    T, K, F = 3, 20, 13
    x = torch.ones(T, K, dtype=BF16, device=dev)
    x[1, 4] = math.inf
    w = torch.full((F, K), 0.5, dtype=BF16, device=dev)
    wd = torch.full((K, F), 0.5, dtype=BF16, device=dev)
    for save in (False, True):           # the kernels for a few tokens, and the tiles
        y = gf.gated_ffn(x, w, w, wd, checkpoint=save)
        y = y[0] if save else y
        assert torch.isinf(y[1]).all() and torch.isfinite(y[[0, 2]]).all()


def test_rows_past_32_bits(dev):
    """More than 2^31 elements: the last rows are what the same rows give alone. (The block's
    products take other tiles and splits then, so that their sums' order differs.)"""
    T, F = 270_000, 8192
    x = torch.zeros(T, F, dtype=BF16, device=dev)
    tail = _randn(dev, 300, F, seed=1).to(BF16)
    x[-300:] = tail
    c = gf.checkpoint8(x)
    alone = gf.checkpoint8(tail)
    assert torch.equal(c.codes[-300:], alone.codes) and torch.equal(c.exponents[-300:],
                                                                    alone.exponents)
    assert torch.equal(c.decode()[-300:], alone.decode())
    w = 1 + 0.3 * _randn(dev, F, seed=2)
    n = gf.rms_norm(x, w, checkpoint=True)
    m = gf.rms_norm(tail, w, checkpoint=True)
    assert torch.equal(n.y[-300:], m.y) and torch.equal(n.checkpoint.codes[-300:],
                                                        m.checkpoint.codes)
    dx, _ = gf.rms_norm_backward(x, n.checkpoint, n.rstd, w)
    assert torch.equal(dx[-300:], gf.rms_norm_backward(tail, m.checkpoint, m.rstd, w)[0])
    del x, c, n, dx
    K = 64
    _, wg, wu, wd, _ = _ffn_inputs(dev, 8, K, F)
    x = torch.zeros(T, K, dtype=BF16, device=dev)
    x[-300:] = tail[:, :K]
    y, s = gf.gated_ffn(x, wg, wu, wd, checkpoint=True)
    ya, sa = gf.gated_ffn(x[-300:], wg, wu, wd, checkpoint=True)

    def near(p, q):
        return (p.double() - q.double()).norm() <= 2 * ROUND * q.double().norm()

    assert near(y[-300:], ya) and not y[:-300].any()
    last = gf.Checkpoint8(s[1].codes[-300:], s[1].exponents[-300:])
    assert near(last.decode(), sa[1].decode())
    g = gf.gated_ffn_backward(x, x, s, wg, wu, wd)
    ga = gf.gated_ffn_backward(x[-300:], x[-300:], sa, wg, wu, wd)
    assert near(g[0][-300:], ga[0])
    assert all(near(p, q) for p, q in zip(g[1:], ga[1:]))     # the other rows add zeros


# ------------------------------------------------------------------ streams, graphs, autograd
def test_streams(dev):
    T, K, F = 300, 256, 520
    x, wg, wu, wd, dy = _ffn_inputs(dev, T, K, F)
    w = torch.ones(K, device=dev)

    def once(stream=None):
        n = gf.rms_norm(x, w, checkpoint=True, stream=stream)
        y, saved = gf.gated_ffn(n.y, wg, wu, wd, checkpoint=True, stream=stream)
        g = gf.gated_ffn_backward(dy, n.checkpoint, saved, wg, wu, wd, gain=w, stream=stream)
        d = gf.rms_norm_backward(g[0], n.checkpoint, n.rstd, w, dh=dy, stream=stream)
        return [y, *g, *d, gf.checkpoint8(y, stream=stream).decode(stream=stream)]

    want = once()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = once(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    with torch.cuda.stream(side):
        got = once()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = once()
    for _ in range(4):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, held))
        assert all(torch.equal(p, q) for p, q in zip(want, once()))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_module_against_float64_autograd(dev, act):
    T, K, F = 96, 128, 200
    torch.manual_seed(0)
    ff = gf.FeedForward(K, F, activation=act, device=dev)
    x = _randn(dev, T, K, seed=1).to(BF16).requires_grad_(True)
    r = _randn(dev, T, K, seed=2).to(BF16).requires_grad_(True)
    dy, dh = _randn(dev, T, K, seed=3).to(BF16), _randn(dev, T, K, seed=4).to(BF16)
    y, h = ff(x, r)
    torch.autograd.backward([y, h], [dy, dh])
    ref = [t.detach().to(F64).requires_grad_(True) for t in
           (x, r, ff.norm, ff.w_gate, ff.w_up, ff.w_down)]
    xr, rr, nw, wg, wu, wd = ref
    hr = xr + rr
    n = hr * (hr.pow(2).mean(1, keepdim=True) + ff.eps) ** -0.5 * nw
    yr = (_act64(n @ wg.t(), act) * (n @ wu.t())) @ wd.t()
    torch.autograd.backward([yr, hr], [dy.to(F64), dh.to(F64)])
    # 8-bit factors (a hundredth each) and bfloat16 products: 3 % of the norm
    for got, want in ((y, yr), (h, hr), (x.grad, xr.grad), (r.grad, rr.grad),
                      (ff.norm.grad, nw.grad), (ff.w_gate.grad, wg.grad),
                      (ff.w_up.grad, wu.grad), (ff.w_down.grad, wd.grad)):
        err = (got.to(F64) - want).norm() / want.norm()
        assert err.item() < 0.03
    y1, h1 = ff(x)
    assert torch.equal(h1, x)
    y1.sum().backward()


def test_module_trains_with_gefen(dev):
    """The block under the library's own optimizer: the loss of a small regression falls."""
    torch.manual_seed(0)
    ff = gf.FeedForward(64, 128, device=dev)
    teacher = gf.FeedForward(64, 128, device=dev)
    opt = gf.Gefen(ff.parameters(), lr=2e-3, weight_decay=0.0)
    x = _randn(dev, 512, 64, seed=1).to(BF16)
    with torch.no_grad():
        target = teacher(x)[0].float()
    losses = []
    for _ in range(60):
        opt.zero_grad()
        loss = (ff(x)[0].float() - target).square().mean()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    assert losses[-1] < 0.5 * losses[0]


def test_saved_bytes(dev):
    """What the block keeps for its backward pass: a byte per normalised element and two per
    inner element, plus exponents and one float per row, beside the parameters."""
    T, K, F = 256, 512, 1024
    ff = gf.FeedForward(K, F, device=dev)
    x = _randn(dev, T, K, seed=1).to(BF16).requires_grad_(True)
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (kept.append(t), t)[1], lambda t: t):
        ff(x)
    rows = [t for t in kept if t.shape[0] == T]
    assert sum(t.numel() * t.element_size() for t in rows) == \
        T * (K + K // 64 + 2 * (F + F // 64) + 4)


# ------------------------------------------------------------------ refusals
def test_refusals(dev):
    x = _randn(dev, 4, 64).to(BF16)
    w = torch.ones(64, device=dev)
    wg, wd = _randn(dev, 32, 64).to(BF16), _randn(dev, 64, 32).to(BF16)
    for bad, err in ((x.half(), TypeError), (x.cpu(), ValueError), ("x", ValueError)):
        with pytest.raises(err):
            gf.checkpoint8(bad)
        with pytest.raises(err):
            gf.rms_norm(bad, w)
        with pytest.raises(err):
            gf.gated_ffn(bad, wg, wg, wd)
    with pytest.raises(TypeError):
        gf.rms_norm(x, w.to(BF16))
    with pytest.raises(ValueError):
        gf.rms_norm(x, w[:63])
    with pytest.raises(ValueError):
        gf.rms_norm(x, w, residual=x[:3])
    with pytest.raises(TypeError):
        gf.rms_norm(x, w, residual=x.float())
    with pytest.raises(gf.GefenError, match="EINVAL"):
        gf.rms_norm(x, w, eps=-1.0)
    with pytest.raises(gf.GefenError, match="EINVAL"):
        gf.rms_norm(x, w, eps=math.nan)
    with pytest.raises(gf.GefenError, match="EINVAL"):
        gf.rms_norm(torch.zeros(1, 16385, device=dev), torch.zeros(16385, device=dev))
    out = gf.rms_norm(x, w, checkpoint=True)
    with pytest.raises(ValueError):
        gf.rms_norm_backward(x[:3], out.checkpoint, out.rstd[:3], w)
    with pytest.raises(ValueError):
        gf.rms_norm_backward(x, out.checkpoint, out.rstd[:3], w)
    with pytest.raises(TypeError):
        gf.gated_ffn(x.float(), wg, wg, wd)
    with pytest.raises(ValueError):
        gf.gated_ffn(x, wg, wg[:31], wd)
    with pytest.raises(ValueError):
        gf.gated_ffn(x, wg[:, :63], wg, wd)
    with pytest.raises(ValueError):
        gf.gated_ffn(x, wg, wg, wd.t())
    with pytest.raises(ValueError):
        gf.gated_ffn(x, wg, wg, wd, activation="relu")
    _, saved = gf.gated_ffn(x, wg, wg, wd, checkpoint=True)
    with pytest.raises(ValueError):
        gf.gated_ffn_backward(x, x, saved, wg, wg, wd, gain=w)
    with pytest.raises(ValueError):
        gf.gated_ffn_backward(x, out.checkpoint, (saved[0], out.checkpoint), wg, wg, wd)
    with pytest.raises(ValueError):
        gf.gated_ffn_backward(x[:3], x[:3], saved, wg, wg, wd)
    with pytest.raises(TypeError):
        gf.Checkpoint8(saved[0].codes.view(torch.uint8), saved[0].exponents)
    with pytest.raises(ValueError):
        gf.Checkpoint8(saved[0].codes, saved[0].exponents[:3])
    with pytest.raises(ValueError):
        saved[0].decode(gain=w[:31])
    with pytest.raises(TypeError):
        saved[0].decode(torch.float16)


def test_example_runs(dev):
    """The example, small: training lowers the loss, serving agrees with training."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "train_feed_forward.py")
    spec = importlib.util.spec_from_file_location("train_feed_forward", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    first, last, err = mod.main(["--layers", "2", "--width", "128", "--inner", "256",
                                 "--tokens", "512", "--steps", "40"])
    assert last < 0.8 * first and err < 2 * ROUND
