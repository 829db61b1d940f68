"""The feed-forward operators that their speed is measured on, through the public entry points.

A training program runs the feed-forward half of a transformer block as: the residual's
addition and RMS norm, the gated feed-forward block, and their backward passes from what the
forward pass saved in 8 bits; a serving program runs the same forward pass on one token or a
prompt and saves nothing. Shapes are those of the Llama-3 1.5B configuration (2048 wide, 8192
inside), the GPT-2 width of 768, the tiny configuration (512, 256), or odd.

Each case is a dict: ``op`` names what is called, the rest its sizes and types.
"""
from __future__ import annotations

import math

import torch

own = False
GROUP = 64
EPS = 1e-6


# ------------------------------------------------------------------------ the cases
def listed():
    return [
        # one token's hidden state into an 8-bit checkpoint and back: the time of the calls
        {"name": "checkpoint_one_token", "op": "checkpoint", "rows": 1, "cols": 2048,
         "dtype": "bf16"},
        # the inner activations of a training batch
        {"name": "checkpoint_8192x8192", "op": "checkpoint", "rows": 8192, "cols": 8192,
         "dtype": "bf16"},
        # serving: the norm of one new token, with the residual
        {"name": "norm_one_token", "op": "norm", "rows": 1, "cols": 2048, "dtype": "bf16",
         "residual": True, "save": False},
        # training: a batch of 8192 tokens, its normalised rows saved in 8 bits
        {"name": "norm_8192x2048_saved", "op": "norm", "rows": 8192, "cols": 2048,
         "dtype": "bf16", "residual": True, "save": True},
        # float32 rows of an odd width that is no multiple of a vector or a group
        {"name": "norm_1000x1601_f32", "op": "norm", "rows": 1000, "cols": 1601, "dtype": "f32",
         "residual": False, "save": True},
        # the norm's backward pass from 8-bit codes, with the residual stream's gradient
        {"name": "norm_backward_8192x2048", "op": "norm_backward", "rows": 8192, "cols": 2048,
         "dtype": "bf16", "residual": True, "save": True},
        # the same from the float32 rows themselves, at the GPT-2 width
        {"name": "norm_backward_1023x768_f32", "op": "norm_backward", "rows": 1023, "cols": 768,
         "dtype": "f32", "residual": False, "save": False},
        # serving one token: the weights' bandwidth
        {"name": "ffn_one_token", "op": "ffn", "tokens": 1, "width": 2048, "inner": 8192,
         "act": "silu"},
        # serving a prompt
        {"name": "ffn_prompt_1000", "op": "ffn", "tokens": 1000, "width": 2048, "inner": 8192,
         "act": "silu"},
        # a training step's forward and backward pass at the tiny configuration
        {"name": "ffn_train_64_tiny", "op": "ffn_train", "tokens": 64, "width": 512,
         "inner": 256, "act": "silu", "saved_input": False},
        # sizes that fit no tile, vector or group, GPT-2's activation
        {"name": "ffn_train_odd", "op": "ffn_train", "tokens": 777, "width": 765, "inner": 2047,
         "act": "gelu", "saved_input": True},
        # a training step of the Llama-3 1.5B feed-forward block, everything saved in 8 bits
        {"name": "ffn_train_8192", "op": "ffn_train", "tokens": 8192, "width": 2048,
         "inner": 8192, "act": "silu", "saved_input": True},
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def _width(rng, lo, hi):
    """Mostly whole heads of 64, else any size."""
    v = _log_int(rng, lo, hi)
    if rng.random() < 0.6:
        v = max(64, 64 * ((v + 32) // 64))
    return v + 64 if v == 3072 else v


def draw(rng):
    op = rng.choice(["checkpoint", "norm", "norm", "norm_backward", "norm_backward", "ffn",
                     "ffn", "ffn_train", "ffn_train", "ffn_train"])
    if op in ("checkpoint", "norm", "norm_backward"):
        rows, cols = _log_int(rng, 1, 16_384), _width(rng, 64, 8192)
        rows = min(rows, 8192 * 8192 // cols)
        case = {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "bf16", "f32"])}
        if op != "checkpoint":
            case.update(residual=rng.random() < 0.6, save=rng.random() < 0.6)
        return case
    if op == "ffn":
        tokens, width, inner = _log_int(rng, 1, 4096), _width(rng, 256, 2048), _width(rng, 256, 8192)
        return {"op": op, "tokens": tokens, "width": width, "inner": inner,
                "act": rng.choice(["silu", "gelu"])}
    tokens, width, inner = _log_int(rng, 16, 8192), _width(rng, 256, 2048), _width(rng, 256, 8192)
    return {"op": op, "tokens": tokens, "width": width, "inner": inner,
            "act": rng.choice(["silu", "gelu"]), "saved_input": rng.random() < 0.6}


# ------------------------------------------------------------------------ the inputs
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _hidden(gen, rows, cols):
    """Hidden states: noise times a scale per channel, a few channels four times as large."""
    scale = torch.exp(0.2 * torch.randn(cols, generator=gen, device="cuda"))
    scale = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.005, 4.0, scale)
    return torch.randn(rows, cols, generator=gen, device="cuda") * scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] in ("checkpoint", "norm", "norm_backward"):
        rows, cols, dt = case["rows"], case["cols"], _DTYPES[case["dtype"]]
        x = _hidden(gen, rows, cols)
        if case["op"] == "checkpoint":
            return dict(s, x=x.to(dt))
        s["weight"] = 1.0 + 0.2 * torch.randn(cols, generator=gen, device="cuda")
        if case["op"] == "norm":
            s["x"] = x.to(dt)
            s["r"] = torch.randn(rows, cols, generator=gen, device="cuda").to(dt) \
                if case["residual"] else None
            return s
        h = x.to(dt)
        s["rstd"] = torch.rsqrt(h.float().square().mean(1) + EPS)
        s["dy"] = (1e-2 * torch.randn(rows, cols, generator=gen, device="cuda")).to(dt)
        s["dh"] = (1e-2 * torch.randn(rows, cols, generator=gen, device="cuda")).to(dt) \
            if case["residual"] else None
        if case["save"]:
            s["codes"], s["exponents"] = _encode(h.float() * s["rstd"][:, None])
        else:
            s["h"] = h
        return s
    tokens, width, inner = case["tokens"], case["width"], case["inner"]
    bf16 = torch.bfloat16

    def weight(rows, cols):
        w = torch.randn(rows, cols, generator=gen, device="cuda")
        return w.mul_(cols ** -0.5).to(bf16)

    n = _hidden(gen, tokens, width)
    n *= torch.rsqrt(n.square().mean(1, keepdim=True) + EPS)
    s["gain"] = 1.0 + 0.2 * torch.randn(width, generator=gen, device="cuda")
    s["x"] = (n * s["gain"]).to(bf16)
    s["w_gate"], s["w_up"] = weight(inner, width), weight(inner, width)
    s["w_down"] = weight(width, inner)
    if case["op"] == "ffn_train":
        s["dy"] = (1e-2 * torch.randn(tokens, width, generator=gen, device="cuda")).to(bf16)
        if case["saved_input"]:
            s["codes"], s["exponents"] = _encode(n)   # as the norm before the block saved them
    return s


# ------------------------------------------------------------------------ the plain form
def _encode(v):
    """Codes and exponents of float32 rows: per group of 64 the smallest power of two that
    keeps the rounded codes within 127, at least 2^-126."""
    rows, cols = v.shape
    groups = -(-cols // GROUP)
    g = torch.nn.functional.pad(v, (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    bits = g.abs().amax(2).view(torch.int32)
    e = (((bits + 0x10000) >> 23) - 6).clamp(min=1)
    codes = torch.round(g / (e << 23).view(torch.float32)[:, :, None])
    return (codes.view(rows, groups * GROUP)[:, :cols].to(torch.int8).contiguous(),
            e.to(torch.uint8))


def _decode(codes, exponents):
    scale = (exponents.to(torch.int32) << 23).view(torch.float32)
    return codes.float() * scale.repeat_interleave(GROUP, 1)[:, :codes.shape[1]]


def _act(g, act):
    """The activation and its derivative, float32."""
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 0.134145 * g * g)


def _plain(s):
    op = s["op"]
    bf16 = torch.bfloat16
    if op == "checkpoint":
        return _decode(*_encode(s["x"].float())).to(bf16)
    if op == "norm":
        dt = s["x"].dtype
        h = s["x"].float()
        if s["r"] is not None:
            h = h + s["r"].float()
        rstd = torch.rsqrt(h.square().mean(1) + EPS)
        n = h * rstd[:, None]
        out = {"y": (n * s["weight"]).to(dt), "rstd": rstd}
        if s["r"] is not None:
            out["h"] = h.to(dt)
        if s["save"]:
            out["saved"] = _decode(*_encode(n)).to(bf16)
        return out
    if op == "norm_backward":
        dt = s["dy"].dtype
        rstd = s["rstd"][:, None]
        n = _decode(s["codes"], s["exponents"]) if s["save"] else s["h"].float() * rstd
        dy = s["dy"].float()
        dn = dy * s["weight"]
        dx = rstd * (dn - n * (dn * n).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(dt), "dweight": (dy * n).sum(0)}
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = x @ wg.t(), x @ wu.t()
    y = ((_act(g, s["act"])[0] * u) @ wd.t()).to(bf16)
    if op == "ffn":
        return y
    gh, uh = _decode(*_encode(g)), _decode(*_encode(u))
    del g, u
    if s["saved_input"]:
        x = _decode(s["codes"], s["exponents"]) * s["gain"]
    dy = s["dy"].float()
    da = dy @ wd
    a, slope = _act(gh, s["act"])
    dg, du = da * uh * slope, da * a
    return {"y": y, "dx": (dg @ wg + du @ wu).to(bf16), "dw_gate": (dg.t() @ x).to(bf16),
            "dw_up": (du.t() @ x).to(bf16), "dw_down": (dy.t() @ (a * uh)).to(bf16)}


# ------------------------------------------------------------------------ the calls
def _own(s):
    import paper_2606_13894_amd as gf
    op = s["op"]
    if op == "checkpoint":
        return gf.checkpoint8(s["x"]).decode()
    if op == "norm":
        r = gf.rms_norm(s["x"], s["weight"], residual=s["r"], eps=EPS, checkpoint=s["save"])
        out = {"y": r.y, "rstd": r.rstd}
        if s["r"] is not None:
            out["h"] = r.h
        if s["save"]:
            out["saved"] = r.checkpoint.decode()
        return out
    if op == "norm_backward":
        saved = gf.Checkpoint8(s["codes"], s["exponents"]) if s["save"] else s["h"]
        dx, dw = gf.rms_norm_backward(s["dy"], saved, s["rstd"], s["weight"], dh=s["dh"])
        return {"dx": dx, "dweight": dw}
    w = (s["w_gate"], s["w_up"], s["w_down"])
    if op == "ffn":
        return gf.gated_ffn(s["x"], *w, activation=s["act"])
    y, saved = gf.gated_ffn(s["x"], *w, activation=s["act"], checkpoint=True)
    x, gain = s["x"], None
    if s["saved_input"]:
        x, gain = gf.Checkpoint8(s["codes"], s["exponents"]), s["gain"]
    dx, dg, du, dd = gf.gated_ffn_backward(s["dy"], x, saved, *w, activation=s["act"], gain=gain)
    return {"y": y, "dx": dx, "dw_gate": dg, "dw_up": du, "dw_down": dd}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------ 64 bits
def _power64(e):
    """2^e for whole e, from its bits (a device's power function may be a bit off)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _saved64(v):
    """What an 8-bit checkpoint of float64 rows stands for."""
    out = torch.empty_like(v)
    for c in range(0, v.shape[1], GROUP):
        block = v[:, c:c + GROUP]
        m, e = torch.frexp(block.abs().amax(1, keepdim=True))   # absmax = m 2^e, m in [1/2, 1)
        e = torch.where(m >= 127.5 / 128, e - 6, e - 7).clamp(min=-126)
        step = _power64(e)
        out[:, c:c + GROUP] = torch.round(block / step) * step
    return out


def _codes64(s):
    step = _power64(s["exponents"].to(torch.int64) - 127)
    return s["codes"].double() * step.repeat_interleave(GROUP, 1)[:, :s["codes"].shape[1]]


def _act64(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    return g / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def _slope64(g, act):
    if act == "silu":
        p = 1 / (1 + torch.exp(-g))
        return p + g * p * (1 - p)
    c = 2 * math.sqrt(2 / math.pi)
    p = 1 / (1 + torch.exp(-c * (g + 0.044715 * g ** 3)))
    return p + g * p * (1 - p) * c * (1 + 3 * 0.044715 * g * g)


def exact(case, seed):
    if "tokens" in case and 18.0 * case["tokens"] * case["width"] * case["inner"] > 4e14:
        return None
    s = prepare(case, seed)
    op = case["op"]
    if op == "checkpoint":
        return _saved64(s["x"].double())
    if op == "norm":
        h = s["x"].double() + (s["r"].double() if s["r"] is not None else 0.0)
        rstd = (h.pow(2).sum(1) / h.shape[1] + EPS) ** -0.5
        n = h * rstd[:, None]
        out = {"y": n * s["weight"].double(), "rstd": rstd}
        if s["r"] is not None:
            out["h"] = h
        if s["save"]:
            out["saved"] = _saved64(n)
        return out
    if op == "norm_backward":
        rstd = s["rstd"].double()[:, None]
        n = _codes64(s) if s["save"] else s["h"].double() * rstd
        dy = s["dy"].double()
        dn = dy * s["weight"].double()
        dot = (dn * n).sum(1, keepdim=True) / n.shape[1]
        dx = rstd * dn - rstd * n * dot
        if s["dh"] is not None:
            dx = dx + s["dh"].double()
        return {"dx": dx, "dweight": (dy * n).sum(0)}
    x, wg, wu, wd = (s[k].double() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
    y = torch.mm(_act64(g, case["act"]) * u, wd.t())
    if op == "ffn":
        return y
    g, u = _saved64(g), _saved64(u)
    xs = _codes64(s) * s["gain"].double() if case["saved_input"] else x
    dy = s["dy"].double()
    da = torch.mm(dy, wd)
    dg = da * u * _slope64(g, case["act"])
    du = da * _act64(g, case["act"])
    return {"y": y, "dx": torch.mm(dg, wg) + torch.mm(du, wu), "dw_gate": torch.mm(dg.t(), xs),
            "dw_up": torch.mm(du.t(), xs), "dw_down": torch.mm(dy.t(), _act64(g, case["act"]) * u)}


# ------------------------------------------------------------------------ what a pass needs
def work(case):
    op = case["op"]
    if "rows" in case:
        n = case["rows"] * case["cols"]
        size = 4 if case["dtype"] == "f32" else 2
        saved = n + case["rows"] * -(-case["cols"] // GROUP)
        if op == "checkpoint":                   # read, write codes, read them, write bfloat16
            return {"bytes": n * (size + 2) + 2 * saved, "flops": 4 * n}
        small = 4 * case["cols"] + 4 * case["rows"]
        if op == "norm":
            streams = 4 if case["residual"] else 2          # x, y; with the residual r and h too
            return {"bytes": n * size * streams + small + (2 * saved + 2 * n if case["save"] else 0),
                    "flops": 8 * n}
        streams = 3 if case["residual"] else 2              # dy, dx; dh
        return {"bytes": n * size * streams + (saved if case["save"] else n * size) + 2 * small,
                "flops": 10 * n}
    t, k, f = case["tokens"], case["width"], case["inner"]
    weights = 6 * k * f
    if op == "ffn":
        return {"bytes": weights + 4 * t * k, "flops": 6 * t * k * f}
    saved = 2 * t * (f + -(-f // GROUP))                    # written once and read once
    x = t * (k + -(-k // GROUP)) if case["saved_input"] else 0
    return {"bytes": 2 * weights + 8 * t * k + 2 * saved + x, "flops": 18 * t * k * f}
