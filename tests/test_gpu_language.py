"""The operators at a language model's two ends (embedding, dropout, token log probabilities, output
head) on the device against float64 formulas.

Bounds. Rounding to bfloat16 moves a value by at most 2^-8 of it, to float32 by 2^-24. A float32 sum
of n terms is off by at most n 2^-24 of the sum of their magnitudes. An exponential of d = z - m in
float32 is off by a relative 2^-24 |d| for the difference, 1.5 * 2^-24 |d| for the product with log2 e
and its rounding, and 2 units in the last place, together taken as (4 |d| + 8) 2^-24. A row's sum
passes through at most V / 256 + 64 additions (a lane's, the lanes', the parts')."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

gf = pytest.importorskip("paper_2606_13894_amd")

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
ROUND = 2.0 ** -8
UNIT = 2.0 ** -24
DTYPES = {"bf16": BF16, "f32": F32}
HALF = {BF16: ROUND, F32: UNIT}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    return torch.device("cuda", 0)


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _randn(dev, *shape, seed=0, dtype=F32):
    return torch.randn(*shape, generator=_gen(dev, seed), device=dev).to(dtype)


def _randint(dev, lo, hi, n, seed=0):
    return torch.randint(lo, hi, (n,), generator=_gen(dev, seed), device=dev)


def _within(got, want, bound, what):
    # what lies past the result's type rounds to infinity: the difference of float32's largest and
    # lowest value, say, which is 6.8e38
    past = want.abs() > torch.finfo(got.dtype).max
    want = torch.where(past, want.sign().to(F64) * math.inf, want.to(F64))
    got = got.to(F64)
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    same = (got == want) | torch.isnan(want)          # infinities among them
    over = torch.where(same, torch.zeros_like(want), (got - want).abs() - bound)
    assert over.numel() == 0 or over.max().item() <= 0.0, (what, over.max().item())


# ------------------------------------------------------------------ embedding
@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("table,out", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"),
                                       ("bf16", "f32")])
@pytest.mark.parametrize("n,vocab,width", [(0, 5, 8), (1, 1, 1), (1, 300, 2048), (7, 5, 3),
                                           (100, 77, 64), (33, 1000, 65), (500, 50, 768),
                                           (9, 20, 2049), (3, 9, 5000)])
def test_embedding(dev, n, vocab, width, table, out, ids):
    w = _randn(dev, vocab, width, seed=1, dtype=DTYPES[table])
    t = _randint(dev, -1, vocab + 1, n, seed=2).to(ids)      # one below 0, one past the end
    y = gf.embedding(t, w, scale=1.75, dtype=DTYPES[out])
    at = t.long().clamp(0, vocab - 1)
    want = (w[at].float() * 1.75).to(DTYPES[out])
    want[t < 0] = 0
    want[t >= vocab] = math.nan
    assert y.dtype is DTYPES[out] and y.shape == (n, width)
    assert torch.equal(torch.nan_to_num(y, nan=7.0), torch.nan_to_num(want, nan=7.0))


def test_embedding_shapes_and_strides(dev):
    w = _randn(dev, 50, 96, seed=1)
    t = _randint(dev, 0, 50, 24, seed=2).view(2, 3, 4)
    y = gf.embedding(t, w)
    assert y.shape == (2, 3, 4, 96) and y.dtype is F32 and torch.equal(y, w[t])
    wide = _randn(dev, 50, 200, seed=3)
    assert torch.equal(gf.embedding(t.transpose(0, 2), wide[:, 7:103]),
                       wide[:, 7:103][t.transpose(0, 2)])
    flat = _randn(dev, 1 + 50 * 96, seed=4)               # a table that starts off 16 bytes
    assert torch.equal(gf.embedding(t, flat[1:].view(50, 96)), flat[1:].view(50, 96)[t])
    assert torch.equal(gf.embedding(t[0, 0, 0], w), w[t[0, 0, 0]])


def _table_gradient(dy, t, vocab, scale):
    """The float64 gradient, the sums of magnitudes, and how many rows each sum has."""
    on = (t >= 0) & (t < vocab)
    at, rows = t[on].long(), dy[on].to(F64) * scale
    zero = torch.zeros(vocab, dy.shape[1], dtype=F64, device=dy.device)
    count = torch.bincount(at, minlength=vocab)[:, None]
    return (zero.index_add(0, at, rows), zero.index_add(0, at, rows.abs()), count)


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"),
                                       ("f32", "bf16")])
@pytest.mark.parametrize("n,vocab,width", [
    (0, 7, 8), (1, 1, 1), (1, 5000, 64), (31, 3, 5), (32, 1, 8), (33, 1, 9), (64, 511, 512),
    (100, 512, 513), (500, 2, 64), (1000, 513, 100), (1000, 40, 2048), (5000, 1000, 72),
    (777, 50257, 768), (3000, 300_001, 8), (20000, 17, 33), (65_537, 100, 16),
    (1024, 3, 24), (1025, 3, 24), (1024, 70_000, 520), (900, 1, 600), (2500, 128_256, 40),
    (20_480, 700, 8), (20_481, 700, 8), (24_576, 50257, 24), (70_001, 300_001, 9),
    (300_000, 5, 16), (1_100_000, 3000, 3)])
def test_embedding_backward(dev, n, vocab, width, dtype, out):
    dy = _randn(dev, n, width, seed=1, dtype=DTYPES[dtype])
    # as text has them: few tokens often
    u = torch.rand(n, generator=_gen(dev, 2), device=dev, dtype=F64)
    t = (torch.exp(u * math.log(vocab + 2)).long() - 2).clamp(-1, vocab)
    g = gf.embedding_backward(dy, t, vocab, scale=0.625, dtype=DTYPES[out])
    want, size, count = _table_gradient(dy, t, vocab, 0.625)
    assert g.dtype is DTYPES[out] and g.shape == (vocab, width)
    _within(g, want, (count + 1) * UNIT * size + HALF[DTYPES[out]] * (want.abs() + UNIT * size),
            "dtable")
    assert not g[count[:, 0] == 0].any()
    again = gf.embedding_backward(dy, t.int(), vocab, scale=0.625, dtype=DTYPES[out])
    assert torch.equal(again, g)


@pytest.mark.parametrize("n", [1000, 4100])
@pytest.mark.parametrize("kind", ["one", "ordered", "turned", "none", "past", "last", "runs",
                                  "around 63"])
def test_embedding_backward_orders(dev, kind, n):
    vocab, width = 3000, 136
    dy = _randn(dev, n, width, seed=1, dtype=BF16)
    i = torch.arange(n, device=dev)
    t = {"one": torch.full_like(i, 1234), "ordered": i.clamp(max=vocab - 1),
         "turned": (n - 1 - i).clamp(max=vocab - 1), "none": torch.full_like(i, -5),
         "past": torch.full_like(i, vocab), "last": torch.full_like(i, vocab - 1),
         "runs": (i // 47) * 31 % vocab,
         # runs of 61 to 67 tokens, as long as the 64 keys that a wave sees and a little more
         "around 63": torch.repeat_interleave(
             torch.arange(70, device=dev), 61 + torch.arange(70, device=dev) % 7)[:n] * 40}[kind]
    g = gf.embedding_backward(dy, t, vocab)
    want, size, count = _table_gradient(dy, t, vocab, 1.0)
    _within(g, want, (count + 2) * UNIT * size, kind)


@pytest.mark.parametrize("n,vocab,width,out", [
    (0, 50_000, 1001, "f32"), (5, 50_000, 1001, "f32"), (1024, 160_001, 517, "bf16"),
    (2000, 160_001, 1037, "bf16"), (21_000, 200_000, 1201, "bf16")])
def test_embedding_backward_of_a_table_with_zeros_apart(dev, n, vocab, width, out):
    """Tables whose zeros take a launch beside the sort's: every row that no token asks for is 0
    whatever was there, also in the last rows and bytes."""
    dtype = DTYPES[out]
    was = torch.full((vocab, width), float("nan"), dtype=dtype, device=dev)
    del was                                       # the memory that the gradient gets
    dy = _randn(dev, n, width, seed=1, dtype=BF16)
    t = _randint(dev, 0, vocab, n, seed=2)
    if n > 3:
        t[1], t[2], t[3] = vocab - 1, 0, vocab - 1
    g = gf.embedding_backward(dy, t, vocab, dtype=dtype)
    used, at = torch.unique(t, return_inverse=True)
    want, size, count = _table_gradient(dy, at, len(used), 1.0)
    _within(g[used], want, (count + 1) * UNIT * size + HALF[dtype] * (want.abs() + UNIT * size),
            "dtable")
    g[used] = 0
    assert not g.any()


def test_embedding_backward_sums_in_order(dev):
    """Few rows of a token are added one by one in increasing position, whatever stands between."""
    dy = _randn(dev, 300, 40, seed=1)
    t = torch.full((300,), -1, device=dev)
    at = [3, 77, 78, 140, 299]
    t[at] = 9
    s = dy[3].clone()
    for i in at[1:]:
        s += dy[i]
    assert torch.equal(gf.embedding_backward(dy, t, 20)[9], s)


# ------------------------------------------------------------------ dropout
def _pieces(n, seed, offset, first=0):
    """16-bit pieces of Philox-4x32-10 from element `first` (a multiple of 8) on."""
    low = np.uint64(0xFFFFFFFF)
    b = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    c = [b & low, b >> np.uint64(32), np.full_like(b, offset & 0xFFFFFFFF),
         np.full_like(b, offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & low,
             (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    words = np.stack(c, 1).astype("<u4").reshape(-1)
    return words.view("<u2")[:n].astype(np.int64)


def test_pieces_are_the_published_generator():
    """Two known answers of Philox-4x32-10 (its authors' test vectors)."""
    def words(p):
        return [int(p[2 * i] | p[2 * i + 1] << 16) for i in range(4)]
    assert words(_pieces(8, 0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 2 ** 64 - 1
    assert words(_pieces(8, ones, ones, first=0)) != words(_pieces(8, 0, 0))


def _dropped(x, p, pieces, residual=None):
    q = round(65536 * p)
    keep = torch.from_numpy(pieces >= q).to(x.device).view(x.shape)
    scale = 65536 / (65536 - q) if q < 65536 else 0.0
    y = torch.where(keep, x.float() * torch.tensor(scale, dtype=F32), 0.0)
    return (y if residual is None else y + residual.float()).to(x.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("shape", [(0,), (1,), (7,), (8,), (9,), (3, 5, 11), (64, 512),
                                   (1000, 777)])
def test_dropout(dev, shape, residual, dtype):
    x = _randn(dev, *shape, seed=1, dtype=DTYPES[dtype])
    r = _randn(dev, *shape, seed=2, dtype=DTYPES[dtype]) if residual else None
    seed, offset = 0x0123456789ABCDEF, (7 << 32) + 5
    pieces = _pieces(x.numel(), seed, offset)
    for p in (0.0, 0.1, 0.5, 65535 / 65536, 1.0):
        want = _dropped(x, p, pieces, r)
        assert torch.equal(gf.dropout(x, p, seed, offset, residual=r), want), p
        state = torch.tensor([seed, offset - 3], device=dev)
        assert torch.equal(gf.dropout(x, p, state, 3, residual=r), want), p


def test_dropout_thresholds(dev):
    """An element is kept up to the p that its piece counts, and dropped from the next step on."""
    x = torch.ones(64, device=dev)
    pieces = _pieces(64, 5, 0)
    for i in (0, 13, 63):
        q = int(pieces[i])
        assert gf.dropout(x, q / 65536, 5)[i].item() > 0
        assert gf.dropout(x, (q + 1) / 65536, 5)[i].item() == 0


def test_dropout_of_infinities(dev):
    """What is dropped is 0 whatever it was; the residual is added as it is."""
    x = torch.full((512,), math.inf, device=dev, dtype=BF16)
    x[::2] = math.nan
    y = gf.dropout(x, 0.5, 1)
    keep = torch.from_numpy(_pieces(512, 1, 0) >= 32768).to(dev)
    assert torch.equal(y == 0, ~keep)
    assert torch.equal(torch.isnan(y), keep & torch.isnan(x))


def test_dropout_strides_and_negative_numbers(dev):
    x = _randn(dev, 40, 60, seed=1)
    t = x.t()
    assert torch.equal(gf.dropout(t, 0.3, 11, 4),
                       _dropped(t.contiguous(), 0.3, _pieces(2400, 11, 4)))
    off = _randn(dev, 1001, seed=2, dtype=BF16)[1:]        # starts off 16 bytes
    assert torch.equal(gf.dropout(off, 0.3, -1, -2),
                       _dropped(off, 0.3, _pieces(1000, 2 ** 64 - 1, 2 ** 64 - 2)))


# ------------------------------------------------------------------ log probabilities
def _rows64(z, t):
    """Float64 results of rows of scores, and the bounds of the float32 ones: lse, logprob,
    entropy and their bounds, log probabilities and theirs."""
    z = z.to(F64)
    V = z.shape[1]
    m = z.amax(1, keepdim=True)
    empty = m == -math.inf
    d = torch.where(empty, -math.inf, z - torch.where(empty, 0.0, m))
    e = d.exp()
    s = e.sum(1, keepdim=True)
    logs = s.log()
    lse = torch.where(empty, -math.inf, m + logs)
    p = torch.where(empty, 0.0, e / s)
    lp = torch.where(empty, -math.inf, d - logs)
    plp = torch.where(p > 0, p * lp, 0.0)
    H = -plp.sum(1)
    H = torch.where(torch.isnan(s[:, 0]), math.nan, H)
    far = torch.where(p > 0, p * d.abs(), 0.0)                  # |d| under p
    far2 = torch.where(p > 0, p * d * d, 0.0)
    adds = (V / 256 + 64) * UNIT
    rel = far.sum(1) * 4 * UNIT + 8 * UNIT + adds
    b_logs = rel + 4 * UNIT * logs[:, 0].abs() + UNIT
    b_lse = b_logs + UNIT * lse.abs()[:, 0]
    b_H = b_logs + 4 * UNIT * far2.sum(1) + (8 * UNIT + adds + 2 * rel + 4 * UNIT) * far.sum(1) \
        + 2 * UNIT * H.abs()
    on = (t >= 0) & (t < V)
    at = t.long().clamp(0, V - 1)[:, None]
    logprob = lp.gather(1, at)[:, 0]
    b_lp = b_logs[:, None] + 2 * UNIT * d.abs() + UNIT * lp.abs()
    b_logprob = b_lp.gather(1, at)[:, 0]
    logprob = torch.where(on, logprob, torch.where(t < 0, 0.0, math.nan))
    return dict(lse=lse[:, 0], H=H, logprob=logprob, b_lse=b_lse, b_H=b_H, b_logprob=b_logprob,
                lp=lp, b_lp=b_lp, p=p, d=d)


def _check_rows(r, want, top=0):
    for name, key in (("logprob", "logprob"), ("entropy", "H"), ("lse", "lse")):
        _within(getattr(r, name), want[key], torch.nan_to_num(want["b_" + key], nan=0.0), name)
    if top:
        v, at = torch.sort(torch.nan_to_num(want["lp"], nan=-math.inf, neginf=-math.inf), dim=1,
                           descending=True, stable=True)
        bad = torch.isnan(want["lse"])
        at = torch.where(bad[:, None], -1, at[:, :top])
        assert torch.equal(r.top_tokens, at)
        _within(r.top_logprobs, torch.where(bad[:, None], math.nan, v[:, :top]),
                want["b_lp"].gather(1, at.clamp(min=0)), "top_logprobs")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,top", [
    (1, 1, 1), (1, 7, 7), (2, 8, 3), (3, 33, 32), (5, 100, 0), (1, 5000, 20), (7, 2048, 5),
    (1, 128_256, 20), (3, 128_256, 32), (1500, 1003, 4), (1100, 50257, 1), (64, 50257, 8),
    (2000, 64, 32), (0, 9, 2), (2, 1_000_003, 20), (600, 270_000, 3)])
def test_token_logprobs(dev, rows, vocab, top, dtype):
    z = _randn(dev, rows, vocab, seed=1).mul_(3).to(DTYPES[dtype])
    t = _randint(dev, -1, vocab + 1, rows, seed=2)
    r = gf.token_logprobs(z, t, top=top)
    if rows:
        # (equal scores have equal log probabilities in float64 too, so the sort's ties are these)
        _check_rows(r, _rows64(z, t), top)
    if not top:
        assert r.top_logprobs is None and r.top_tokens is None
    again = gf.token_logprobs(z, t.int(), top=top)
    for a, b in zip(r, again):
        assert a is None and b is None or torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(1, 20000), (40, 777), (1200, 3001)])
def test_token_logprobs_masks(dev, rows, vocab, dtype):
    """Most scores -inf, rows of one score, rows of nothing, scores at the type's lowest value,
    infinities and NaN, equal scores, zeros of both signs."""
    dt = DTYPES[dtype]
    z = _randn(dev, rows, vocab, seed=1).mul_(2).to(dt)
    z[torch.rand(rows, vocab, generator=_gen(dev, 3), device=dev) < 0.97] = -math.inf
    kinds = {}

    def put(name, row):
        if rows > 1 or name == only:
            kinds[name] = (row % rows)
            return z[row % rows]
        return torch.empty(vocab, device=dev, dtype=dt)

    for only in ([None] if rows > 1 else ["nothing", "one", "lowest", "level", "zeros", "nan",
                                          "inf", "mixed"]):
        put("nothing", 1)[:] = -math.inf
        row = put("one", 2)
        row[:] = -math.inf
        row[vocab - 1] = 3.0
        put("lowest", 3)[:] = torch.finfo(dt).min
        put("level", 4)[:] = 1.5
        row = put("zeros", 5)
        row[:] = 0.0
        row[::2] = -0.0
        put("nan", 6)[vocab // 2] = math.nan
        put("inf", 7)[vocab // 3] = math.inf
        row = put("mixed", 8)
        row[:] = torch.finfo(dt).min
        row[::3] = -math.inf
        row[5] = torch.finfo(dt).max
        t = _randint(dev, 0, vocab, rows, seed=2)
        want = _rows64(z, t)
        bad = torch.isnan(z).any(1) | (z == math.inf).any(1)
        for k in ("lse", "H", "logprob"):
            want[k] = torch.where(bad, math.nan, want[k])
        want["lp"] = torch.where(z == -math.inf, -math.inf, want["lp"])
        for top in (0, 6):
            _check_rows(gf.token_logprobs(z, t, top=top), want, top)
        assert len(kinds) >= 1


def test_top_where_one_lane_holds_the_best(dev):
    """More large scores in one lane's part of a row than the list holds: the k best are taken one
    by one."""
    vocab = 256 * 8 * 200
    z = torch.full((1100, vocab), -5.0, device=dev, dtype=BF16)
    lane = (torch.arange(vocab, device=dev) // 8) % 256
    z[3, lane == 17] = 2.0
    z[4, lane < 31] = 2.0
    z[5, lane == 255] = _randn(dev, 1600, seed=1, dtype=BF16).abs() + 1
    t = torch.zeros(1100, dtype=torch.int64, device=dev)
    r = gf.token_logprobs(z, t, top=32)
    for row in (3, 4, 5, 6):
        at = torch.sort(z[row].float(), descending=True, stable=True)[1][:32]
        assert torch.equal(r.top_tokens[row], at), row


def test_token_logprobs_rows_apart(dev):
    """A vocabulary padded in memory, leading dimensions, rows off 16 bytes: no copy is needed."""
    z = _randn(dev, 4, 30, 520, seed=1, dtype=BF16)
    t = _randint(dev, 0, 501, 120, seed=2).view(4, 30)
    r = gf.token_logprobs(z[..., 3:504], t, top=2)
    dense = gf.token_logprobs(z[..., 3:504].contiguous(), t, top=2)
    for a, b in zip(r, dense):
        assert a.shape[:2] == (4, 30) and torch.equal(a, b)
    one = gf.token_logprobs(z[0, :1, 3:504], t[0, :1], top=2)
    assert torch.equal(one.logprob, r.logprob[0, :1])
    turned = gf.token_logprobs(z[0, :, 3:504].t().contiguous().t(), t[0])
    assert torch.equal(turned.logprob, r.logprob[0])


def _score_gradient64(z, t, lse, H, g, h):
    """The float64 gradient from the forward pass's float32 results, and its bound but for the
    output's rounding."""
    z, lse, H, g, h = (v.to(F64) for v in (z, lse, H, g, h))
    V = z.shape[1]
    empty = (lse == -math.inf)[:, None]
    on = (t >= 0) & (t < V)
    g = torch.where(on, g, 0.0)[:, None]
    d = torch.where(empty, -math.inf, z - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    p = d.exp()
    inner = torch.where(p > 0, d + H[:, None], 0.0)
    dz = -p * (g + h[:, None] * inner)
    size = p * (g.abs() + (h[:, None] * inner).abs())
    near = torch.where(p > 0, d.abs(), 0.0)
    bound = size * (4 * near + 16) * UNIT + p * h.abs()[:, None] * (near + H.abs()[:, None]) * 4 * UNIT
    hit = torch.zeros_like(z, dtype=torch.bool)
    hit[on.nonzero()[:, 0], t[on].long()] = True
    dz = torch.where(empty, 0.0, dz + torch.where(hit, g, 0.0))
    return dz, bound + torch.where(hit, 2 * UNIT * g.abs(), 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 7), (3, 9), (5, 4097), (40, 1000), (2, 128_256),
                                        (300, 50257), (0, 5)])
def test_token_logprobs_backward(dev, rows, vocab, dtype):
    dt = DTYPES[dtype]
    z = _randn(dev, rows, vocab, seed=1).mul_(3).to(dt)
    if vocab > 20 and rows > 4:
        z[0, : vocab // 2] = -math.inf
        z[1] = -math.inf
        z[2] = torch.finfo(dt).min
        z[3, 4] = math.nan
    t = _randint(dev, -1, vocab + 1, rows, seed=2)
    g, h = _randn(dev, rows, seed=3), _randn(dev, rows, seed=4)
    r = gf.token_logprobs(z, t)
    for ent in (h, None):
        got = gf.token_logprobs_backward(g, z, t, r.lse, r.entropy, dentropy=ent)
        assert got.dtype is dt and got.shape == z.shape
        if rows:
            want, bound = _score_gradient64(z, t, r.lse, r.entropy, g,
                                            torch.zeros_like(g) if ent is None else h)
            # values below the smallest normal number may be flushed
            _within(got, want, torch.nan_to_num(bound) + HALF[dt] * want.abs() + 2.0 ** -126,
                    "dlogits")
        again = z.clone()
        assert gf.token_logprobs_backward(g, again, t.int(), r.lse, r.entropy, dentropy=ent,
                                          out=again) is again
        assert torch.equal(torch.nan_to_num(again), torch.nan_to_num(got))


def test_token_logprobs_backward_rows_apart(dev):
    z = _randn(dev, 50, 700, seed=1, dtype=BF16)
    t = _randint(dev, 0, 601, 50, seed=2)
    g = _randn(dev, 50, seed=3)
    part = z[:, 11:612]
    r = gf.token_logprobs(part, t)
    want = gf.token_logprobs_backward(g, part, t, r.lse, r.entropy)
    wide = torch.full((50, 800), 9.0, device=dev, dtype=BF16)
    gf.token_logprobs_backward(g, part, t, r.lse, r.entropy, out=wide[:, 1:602])
    assert torch.equal(wide[:, 1:602], want)
    assert (wide[:, :1] == 9).all() and (wide[:, 602:] == 9).all()
    whole = z.clone()
    gf.token_logprobs_backward(g, whole[:, 11:612], t, r.lse, r.entropy, out=whole[:, 11:612])
    assert torch.equal(whole[:, 11:612], want)
    assert torch.equal(whole[:, :11], z[:, :11]) and torch.equal(whole[:, 612:], z[:, 612:])


# ------------------------------------------------------------------ output head
HEAD_SIZES = [(1, 8, 5), (2, 1, 1), (3, 64, 1), (5, 100, 300), (16, 2048, 1003), (17, 509, 1003),
              (64, 512, 1000), (64, 509, 1003), (130, 72, 2500), (300, 256, 4097), (1000, 765, 3001),
              (2100, 128, 6000)]


def _head64(x, w, t):
    z = x.to(F64) @ w.to(F64).t()
    want = _rows64(z, t)
    # the scores' own error, a float32 sum's
    dz = x.shape[1] * UNIT * (x.to(F64).abs() @ w.to(F64).abs().t()).amax(1)
    want["b_lse"] += dz
    want["b_logprob"] += 2 * dz
    want["b_H"] += 2 * dz * (torch.where(want["p"] > 0, want["p"] * want["lp"].abs(), 0.0).sum(1)
                             + want["H"].abs())
    return z, want, dz


@pytest.mark.parametrize("n,width,vocab", HEAD_SIZES)
def test_head_logprobs(dev, n, width, vocab):
    x = _randn(dev, n, width, seed=1, dtype=BF16)
    w = _randn(dev, vocab, width, seed=2).mul_(2 * width ** -0.5).to(BF16)
    t = _randint(dev, -1, vocab + 1, n, seed=3)
    r = gf.head_logprobs(x, w, t)
    _, want, _ = _head64(x, w, t)
    _check_rows(r, want)
    again = gf.head_logprobs(x, w, t.int())
    for a, b in zip(r, again):
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def _check_head_gradients(x, w, t, g, h, r, dx, dw):
    z, _, dz_err = _head64(x, w, t)
    hh = torch.zeros_like(g) if h is None else h
    want, bound = _score_gradient64(z, t, r.lse, r.entropy, g, hh)
    d = z - r.lse.to(F64)[:, None]
    p = d.exp()
    # a score off by e moves its gradient by at most e p (|g| + |h| (|d| + |H| + 1)) to first
    # order; twice that for what is beyond it
    slope = p * (g.to(F64).abs()[:, None] + hh.to(F64).abs()[:, None] *
                 (d.abs() + r.entropy.to(F64).abs()[:, None] + 1))
    bound = bound + 2 * dz_err[:, None] * slope
    bound = bound + ROUND * (want.abs() + bound) + 2.0 ** -126       # what the products read
    xa, wa = x.to(F64).abs(), w.to(F64).abs()
    ex, ew = want @ w.to(F64), want.t() @ x.to(F64)
    size = want.abs() + bound
    bx = bound @ wa + (w.shape[0] + 16) * UNIT * (size @ wa)
    bw = bound.t() @ xa + (x.shape[0] + 16) * UNIT * (size.t() @ xa)
    _within(dx, ex, bx + ROUND * (ex.abs() + bx), "dx")
    _within(dw, ew, bw + ROUND * (ew.abs() + bw), "dweight")


@pytest.mark.parametrize("n,width,vocab", HEAD_SIZES)
def test_head_logprobs_backward(dev, n, width, vocab):
    x = _randn(dev, n, width, seed=1, dtype=BF16)
    w = _randn(dev, vocab, width, seed=2).mul_(2 * width ** -0.5).to(BF16)
    t = _randint(dev, -1, vocab + 1, n, seed=3)
    g, h = _randn(dev, n, seed=4), _randn(dev, n, seed=5)
    r = gf.head_logprobs(x, w, t)
    for ent in (h, None):
        dx, dw = gf.head_logprobs_backward(g, x, w, t, r.lse, r.entropy, dentropy=ent)
        assert dx.dtype is BF16 and dw.dtype is BF16
        _check_head_gradients(x, w, t, g, ent, r, dx, dw)
    again = gf.head_logprobs_backward(g, x, w, t.int(), r.lse, r.entropy)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("n,width,vocab", [(3, 64, 1000), (64, 509, 1003), (300, 72, 700),
                                           (4500, 64, 140_001)])
def test_head_backward_of_one_gradient(dev, n, width, vocab):
    """One gradient without the other has the bits that both have, through the call and where the
    module's weight, or its input, is frozen."""
    x = _randn(dev, n, width, seed=1, dtype=BF16)
    w = _randn(dev, vocab, width, seed=2).mul_(2 * width ** -0.5).to(BF16)
    t = _randint(dev, -1, vocab, n, seed=3)
    g, h = _randn(dev, n, seed=4), _randn(dev, n, seed=5)
    r = gf.head_logprobs(x, w, t)
    arguments = (g, x, w, t, r.lse, r.entropy, h)
    dx, dw = gf.head_logprobs_backward(*arguments)
    a, none = gf.head_logprobs_backward(*arguments, weight_grad=False)
    assert none is None and torch.equal(a, dx)
    none, b = gf.head_logprobs_backward(*arguments, x_grad=False)
    assert none is None and torch.equal(b, dw)
    with pytest.raises(ValueError, match="neither"):
        gf.head_logprobs_backward(*arguments, x_grad=False, weight_grad=False)
    for of_x in (True, False):
        head = gf.Head(width, vocab, weight=torch.nn.Parameter(w.float(), requires_grad=not of_x))
        leaf = x.clone().requires_grad_(of_x)
        logprob, entropy = head(leaf, t)
        torch.autograd.backward((logprob, entropy), (g, h))
        if of_x:
            assert torch.equal(leaf.grad, dx) and head.weight.grad is None
        else:
            assert torch.equal(head.weight.grad, dw.float()) and leaf.grad is None


@pytest.mark.parametrize("n,width,vocab", [(4500, 64, 140_001), (40_000, 40, 30_000)])
def test_head_backward_by_ranges(dev, n, width, vocab):
    """More gradients of scores than are held at once: ranges of the vocabulary, dx summed over
    them; against a float64 gradient over pieces of it."""
    x = _randn(dev, n, width, seed=1, dtype=BF16)
    w = _randn(dev, vocab, width, seed=2).mul_(2 * width ** -0.5).to(BF16)
    t = _randint(dev, 0, vocab, n, seed=3)
    g = _randn(dev, n, seed=4)
    r = gf.head_logprobs(x, w, t)
    dx, dw = gf.head_logprobs_backward(g, x, w, t, r.lse, r.entropy)
    ex = torch.zeros(n, width, dtype=F64, device=dev)
    bx = torch.zeros_like(ex)
    x64 = x.to(F64)
    for a in range(0, vocab, 10_000):
        wp = w[a:a + 10_000].to(F64)
        z = x64 @ wp.t()
        err = width * UNIT * (x64.abs() @ wp.abs().t()).amax(1)[:, None]
        p = (z - r.lse.to(F64)[:, None]).exp()
        dz = -g.to(F64)[:, None] * p
        bound = dz.abs() * ((4 * (z - r.lse.to(F64)[:, None]).abs() + 20) * UNIT + 2 * err)
        inside = (t >= a) & (t < a + wp.shape[0])
        rows = inside.nonzero()[:, 0]
        dz[rows, t[rows] - a] += g.to(F64)[rows]
        bound = bound + (ROUND + 4 * UNIT) * (dz.abs() + bound)
        ew = dz.t() @ x64
        bw = bound.t() @ x64.abs() + n * UNIT * ((dz.abs() + bound).t() @ x64.abs())
        _within(dw[a:a + 10_000], ew, bw + ROUND * (ew.abs() + bw), f"dweight from {a}")
        ex += dz @ wp
        bx += bound @ wp.abs() + vocab * UNIT * ((dz.abs() + bound) @ wp.abs())
    _within(dx, ex, bx + ROUND * (ex.abs() + bx), "dx")


def test_head_zero_tokens(dev):
    x = torch.empty(0, 64, device=dev, dtype=BF16)
    w = _randn(dev, 100, 64, seed=1, dtype=BF16)
    t = torch.empty(0, dtype=torch.int64, device=dev)
    r = gf.head_logprobs(x, w, t)
    assert r.logprob.shape == (0,)
    e = torch.empty(0, device=dev)
    dx, dw = gf.head_logprobs_backward(e, x, w, t, e, e)
    assert dx.shape == (0, 64) and not dw.any()


def test_head_rows_stay_apart(dev):
    """A row of NaN or infinities is its own trouble; rows off 16 bytes are copied."""
    n, width, vocab = 200, 128, 999
    flat = _randn(dev, n * width + 3, seed=1, dtype=BF16)
    x = flat[3:].view(n, width)
    w = _randn(dev, vocab, width, seed=2).mul_(0.2).to(BF16)
    t = _randint(dev, 0, vocab, n, seed=3)
    clean = gf.head_logprobs(x.clone(), w, t)
    x[7] = math.nan
    x[70, 5] = math.inf
    r = gf.head_logprobs(x, w, t)
    ok = torch.ones(n, dtype=torch.bool, device=dev)
    ok[7] = ok[70] = False
    for a, b in zip(r, clean):
        assert torch.equal(a[ok], b[ok]) and torch.isnan(a[~ok]).all()
    g = _randn(dev, n, seed=4)
    dx, _ = gf.head_logprobs_backward(g, x, w, t, r.lse, r.entropy)
    assert torch.isfinite(dx[ok]).all()


# ------------------------------------------------------------------ a run of them together
def _plain_model(tokens, nxt, table, keep, scale):
    """The same run in float64 under torch's autograd."""
    h = torch.where(keep, table[tokens] * scale, 0.0)
    lp = torch.log_softmax(h @ table.t(), 1)
    taken = lp.gather(1, nxt.clamp(min=0)[:, None])[:, 0]
    return -(torch.where(nxt >= 0, taken, 0.0)).mean(), -(lp.exp() * lp).sum(1).mean()


def test_modules_together(dev):
    """Embedding, dropout and the head over one table, its gradient the sum of both uses, against
    float64. The gradient is off by the roundings of the rows (2^-8, into the head's products and
    scores), of the scores' gradients and of the outputs: 6 of them, in the mean of squares."""
    torch.manual_seed(0)
    vocab, width, n = 301, 96, 500
    emb = gf.Embedding(vocab, width, scale=1.0, device=dev)
    with torch.no_grad():
        emb.table.copy_(_randn(dev, vocab, width, seed=1).to(BF16).float() * 0.25)
    drop = gf.Dropout(0.25, seed=9, device=dev)
    head = gf.Head(width, vocab, weight=emb.table)
    t, nxt = _randint(dev, 0, vocab, n, seed=2), _randint(dev, -1, vocab, n, seed=3)
    assert len(list(torch.nn.ModuleList([emb, drop, head]).parameters())) == 1
    for step in range(2):
        emb.table.grad = None
        logprob, entropy = head(drop(emb(t)), nxt)
        loss = -logprob.mean() - 0.01 * entropy.mean()
        loss.backward()
        keep = torch.from_numpy(_pieces(n * width, 9, step) >= 16384).to(dev).view(n, width)
        w64 = emb.table.detach().to(F64).requires_grad_()
        nll, ent = _plain_model(t, nxt, w64, keep, 65536 / 49152)
        want = nll - 0.01 * ent
        want.backward()
        assert abs(loss.item() - want.item()) <= 4 * ROUND * abs(want.item())
        err = (emb.table.grad.to(F64) - w64.grad).norm() / w64.grad.norm()
        assert err.item() <= 6 ** 0.5 * ROUND, err.item()
    assert drop.state.tolist() == [9, 2]
    drop.eval()
    x = emb(t)
    assert drop(x) is x and drop.state.tolist() == [9, 2]


def test_logprobs_module_matches_differences(dev):
    """The gradient of float32 logits against central differences of float64 results."""
    z = _randn(dev, 3, 50, seed=1).requires_grad_()
    t = torch.tensor([4, 49, -1], device=dev)
    lp, H = gf.LogProbs()(z, t)
    a, b = _randn(dev, 3, seed=2), _randn(dev, 3, seed=3)
    (lp * a + H * b).sum().backward()

    def value(v):
        r = _rows64(v, t)
        return (r["logprob"] * a.to(F64) + r["H"] * b.to(F64)).sum().item()

    step = 2.0 ** -12
    for i, j in ((0, 4), (0, 5), (1, 49), (1, 0), (2, 7)):
        up, down = z.detach().to(F64).clone(), z.detach().to(F64).clone()
        up[i, j] += step
        down[i, j] -= step
        slope = (value(up) - value(down)) / (2 * step)
        # third derivatives are at most about 10 |a| + 30 |b|, and step^2 / 6 of them is left
        size = 10 * abs(a[i].item()) + 30 * abs(b[i].item())
        assert abs(z.grad[i, j].item() - slope) <= step ** 2 / 6 * size + 64 * UNIT * size
    lp, _ = gf.LogProbs()(z, t)        # only one of the results is used
    lp.sum().backward()


def test_second_derivatives_and_plain_calls_are_errors(dev):
    emb = gf.Embedding(20, 64, device=dev)
    head = gf.Head(64, 20, device=dev)
    drop = gf.Dropout(0.5, device=dev)
    t = torch.arange(10, device=dev)
    lp, _ = head(drop(emb(t)), t)
    grads = torch.autograd.grad(lp.sum(), [emb.table, head.weight], create_graph=True)
    for g in grads:
        with pytest.raises(RuntimeError, match="second derivative|cannot be differentiated"):
            g.sum().backward(retain_graph=True)
    w = emb.table
    for y in (gf.embedding(t, w), gf.dropout(w, 0.5, 1), gf.token_logprobs(w, torch.zeros_like(
            torch.arange(20, device=dev))).logprob):
        with pytest.raises(RuntimeError, match="no gradient of its own"):
            y.sum().backward()


# ------------------------------------------------------------------ streams and graphs
def test_on_another_stream(dev):
    t = _randint(dev, 0, 500, 300, seed=1)
    w = _randn(dev, 500, 256, seed=2).to(BF16)
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    x = gf.embedding(t, w, stream=side)
    y = gf.dropout(x, 0.1, 3, stream=side)
    r = gf.head_logprobs(y, w, t, stream=side)
    g = torch.ones(300, device=dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    dx, dw = gf.head_logprobs_backward(g, y, w, t, r.lse, r.entropy, stream=side)
    de = gf.embedding_backward(dx, t, 500, stream=side)
    s = gf.token_logprobs(x, t.clamp(max=255), top=3, stream=side)
    dz = gf.token_logprobs_backward(g, x, t.clamp(max=255), s.lse, s.entropy, stream=side)
    torch.cuda.synchronize()
    x2 = gf.embedding(t, w)
    y2 = gf.dropout(x2, 0.1, 3)
    r2 = gf.head_logprobs(y2, w, t)
    d2 = gf.head_logprobs_backward(g, y2, w, t, r2.lse, r2.entropy)
    s2 = gf.token_logprobs(x2, t.clamp(max=255), top=3)
    assert torch.equal(x, x2) and torch.equal(y, y2) and torch.equal(r.logprob, r2.logprob)
    assert torch.equal(dx, d2[0]) and torch.equal(dw, d2[1])
    assert torch.equal(de, gf.embedding_backward(d2[0], t, 500))
    assert torch.equal(s.top_tokens, s2.top_tokens)
    assert torch.equal(dz, gf.token_logprobs_backward(g, x2, t.clamp(max=255), s2.lse, s2.entropy))


def test_captured_training_step(dev):
    """Forward and backward in a graph, replayed with new tokens and weights between eager calls:
    the results are the eager ones, and dropout goes on with its numbers."""
    torch.manual_seed(0)
    vocab, width, n = 400, 128, 96
    emb = gf.Embedding(vocab, width, device=dev)
    drop = gf.Dropout(0.2, seed=5, device=dev)
    head = gf.Head(width, vocab, device=dev)
    t, nxt = _randint(dev, 0, vocab, n, seed=1), _randint(dev, 0, vocab, n, seed=2)
    params = [emb.table, head.weight]

    def step():
        lp, H = head(drop(emb(t)), nxt)
        loss = -lp.mean() - 0.1 * H.mean()
        return (loss, *torch.autograd.grad(loss, params))

    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream(dev).wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        t.copy_(_randint(dev, 0, vocab, n, seed=10 + k))
        with torch.no_grad():
            emb.table.mul_(1.5)
        at = drop.state.clone()
        graph.replay()
        got = [v.clone() for v in out]
        assert drop.state.tolist() == [5, at[1].item() + 1]
        drop.state.copy_(at)
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), k


def test_captured_accumulation(dev):
    """The same with ``backward``, which adds to the parameters' gradients: two passes in a graph."""
    torch.manual_seed(0)
    vocab, width, n = 300, 64, 50
    emb = gf.Embedding(vocab, width, device=dev)
    drop = gf.Dropout(0.2, seed=5, device=dev)
    head = gf.Head(width, vocab, weight=emb.table, device=dev)
    t, nxt = _randint(dev, -1, vocab, n, seed=1), _randint(dev, -1, vocab, n, seed=2)

    def step():
        emb.table.grad = None
        for _ in range(2):
            (-head(drop(emb(t)), nxt)[0].mean()).backward()

    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.current_stream(dev).wait_stream(side)
    torch.cuda.synchronize()
    emb.table.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    captured = emb.table.grad
    for k in range(3):
        t.copy_(_randint(dev, -1, vocab, n, seed=10 + k))
        at = drop.state.clone()
        graph.replay()
        got = captured.clone()
        drop.state.copy_(at)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, emb.table.grad), k


def test_two_graphs_of_calls(dev):
    """Two captured graphs of the plain calls with workspaces from one pool, replayed in turns."""
    w = _randn(dev, 3000, 256, seed=1).to(BF16)
    big = _randn(dev, 2, 100_000, seed=2)
    ts = [_randint(dev, 0, 3000, 700, seed=3), _randint(dev, 0, 3000, 40, seed=4)]
    g = [_randn(dev, len(t), seed=5) for t in ts]

    def run(i):
        x = gf.embedding(ts[i], w)
        r = gf.head_logprobs(x, w, ts[i])
        dx, dw = gf.head_logprobs_backward(g[i], x, w, ts[i], r.lse, r.entropy)
        s = gf.token_logprobs(big, ts[i][:2], top=5)
        return (r.logprob, dx, dw, gf.embedding_backward(dx, ts[i], 3000), s.logprob,
                s.top_tokens)

    want = [run(0), run(1)]
    torch.cuda.synchronize()
    pool = torch.cuda.graph_pool_handle()
    graphs, outs = [], []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            outs.append(run(i))
        graphs.append(graph)
    for k in range(3):
        for i in (0, 1):
            graphs[i].replay()
            torch.cuda.synchronize()
            for a, b in zip(outs[i], want[i]):
                assert torch.equal(a, b), (k, i)
            run(1 - i)
