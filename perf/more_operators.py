"""The operators at a language model's two ends that their speed is measured on, through the public
entry points.

Around the blocks whose gradients the step takes, a training program looks its tokens up in an
embedding table, drops a part of the activations, and ends in the log probabilities of the tokens
that followed, over the vocabulary; the backward pass gives the gradients of the head's weight and
of the table, the largest tensors of the models here. A serving or scoring program looks up one
token, and asks for the log probability of the token that was taken, the entropy and the best
alternatives. Shapes are those of the Llama-3 1.5B configuration (vocabulary 128256, width 2048),
the GPT-2 one (50257, 768), the tiny one (512 wide), or odd.

Each case is a dict: ``op`` names what is called, the rest its sizes and types.

Dropout's mask is defined by Philox-4x32-10 (Salmon et al., SC 2011): element i takes 16-bit piece
i mod 8 (a word's low half first) of the block with counter (i / 8, offset) and key seed, and is
kept where that is at least round(65536 p).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


# ------------------------------------------------------------------------ the cases
def listed():
    return [
        # serving: the row of one new token, from a table cast once
        {"name": "embed_one_token", "op": "embed", "tokens": 1, "vocab": 128_256, "width": 2048,
         "table": "bf16", "scaled": False, "train": False},
        # a training step at the GPT-2 sizes, its batch padded to an odd length: float32 table and
        # gradient, rows scaled by the root of the width
        {"name": "embed_train_1023x768_f32", "op": "embed", "tokens": 1023, "vocab": 50_257,
         "width": 768, "table": "f32", "scaled": True, "train": True},
        # a training step of the Llama-3 1.5B configuration, bfloat16 gradients as it has them
        {"name": "embed_train_8192x2048", "op": "embed", "tokens": 8192, "vocab": 128_256,
         "width": 2048, "table": "bf16", "scaled": False, "train": True},
        # the tiny configuration's activations, forward and back: the time of the calls
        {"name": "dropout_64x512", "op": "dropout", "rows": 64, "cols": 512, "dtype": "bf16",
         "residual": False, "p": 0.1},
        # the residual branch of a training batch, added to its residual, and back
        {"name": "dropout_8192x2048_residual", "op": "dropout", "rows": 8192, "cols": 2048,
         "dtype": "bf16", "residual": True, "p": 0.1},
        # serving: one row of logits, the taken token with twenty alternatives
        {"name": "logprobs_one_row_top20", "op": "logprobs", "rows": 1, "vocab": 128_256,
         "dtype": "bf16", "top": 20, "masked": False, "train": False},
        # scoring a prompt of 2048 tokens, five alternatives each
        {"name": "logprobs_2048_top5", "op": "logprobs", "rows": 2048, "vocab": 128_256,
         "dtype": "bf16", "top": 5, "masked": False, "train": False},
        # a policy's training step over float32 logits with most tokens ruled out; rows of an odd
        # length
        {"name": "logprobs_train_1023x50257_f32", "op": "logprobs", "rows": 1023, "vocab": 50_257,
         "dtype": "f32", "top": 0, "masked": True, "train": True},
        # scoring one token from its hidden state: the weight's bandwidth
        {"name": "head_one_token", "op": "head", "tokens": 1, "width": 2048, "vocab": 128_256,
         "train": False},
        # scoring a prompt
        {"name": "head_prompt_1000", "op": "head", "tokens": 1000, "width": 2048,
         "vocab": 128_256, "train": False},
        # a small model's training step, sizes that fit no tile or vector
        {"name": "head_train_64_odd", "op": "head", "tokens": 64, "width": 509, "vocab": 1003,
         "train": True},
        # a training step of the Llama-3 1.5B configuration's output head
        {"name": "head_train_8192", "op": "head", "tokens": 8192, "width": 2048,
         "vocab": 128_256, "train": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly whole heads of 64, else any size."""
    v = _log_int(rng, lo, hi)
    return max(64, 64 * ((v + 32) // 64)) if rng.random() < 0.6 else v


def _vocab(rng, lo):
    """Mostly padded to whole multiples of 64, else any size."""
    v = _log_int(rng, lo, 128_256)
    return min(128_256, 64 * ((v + 63) // 64)) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["embed", "embed", "dropout", "logprobs", "logprobs", "head", "head"])
    if op == "embed":
        return {"op": op, "tokens": _log_int(rng, 1, 16_384), "vocab": _vocab(rng, 256),
                "width": _width(rng, 64, 2048), "table": rng.choice(["bf16", "f32"]),
                "scaled": rng.random() < 0.5, "train": rng.random() < 0.7}
    if op == "dropout":
        return {"op": op, "rows": _log_int(rng, 1, 8192), "cols": _width(rng, 64, 8192),
                "dtype": rng.choice(["bf16", "bf16", "f32"]), "residual": rng.random() < 0.5,
                "p": rng.choice([0.05, 0.1, 0.2, 0.5])}
    if op == "logprobs":
        train = rng.random() < 0.5
        return {"op": op, "rows": _log_int(rng, 1, 2048), "vocab": _vocab(rng, 1000),
                "dtype": rng.choice(["bf16", "bf16", "f32"]),
                "top": 0 if train else rng.choice([0, 1, 5, 20]), "masked": rng.random() < 0.3,
                "train": train}
    train = rng.random() < 0.6
    return {"op": op, "tokens": _log_int(rng, 16 if train else 1, 4096),
            "width": _width(rng, 128, 2048), "vocab": _vocab(rng, 256), "train": train}


# ------------------------------------------------------------------------ the inputs
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tokens(gen, n, vocab, ignored=0.0):
    """Tokens as text has them, rank r about 1 / r as often, at ids that are no order of rank; a
    share of them -1: padding, or prompt tokens that no loss is taken on."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * math.log(vocab)).long().clamp(1, vocab) - 1
    t = torch.randperm(vocab, generator=gen, device="cuda")[rank]
    return torch.where(torch.rand(n, generator=gen, device="cuda") < ignored, -1, t)


def _upstream(gen, n):
    """The gradients of a mean over tokens, with a weight for each."""
    w = 0.5 + torch.rand(n, generator=gen, device="cuda")
    e = 0.02 * torch.rand(n, generator=gen, device="cuda")
    return -w / n, e / n


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op = case["op"]

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    if op == "embed":
        n, v, w = case["tokens"], case["vocab"], case["width"]
        s["ids"] = _tokens(gen, n, v, 0.05 if case["train"] and n > 1 else 0.0)
        s["weight"] = randn(v, w).mul_(0.02).to(_DTYPES[case["table"]])
        s["scale"] = math.sqrt(w) if case["scaled"] else 1.0
        if case["train"]:
            s["dy"] = (1e-3 * randn(n, w)).to(torch.bfloat16)
        return s
    if op == "dropout":
        dt = _DTYPES[case["dtype"]]
        s["x"] = randn(case["rows"], case["cols"]).to(dt)
        s["r"] = randn(case["rows"], case["cols"]).to(dt) if case["residual"] else None
        s["dy"] = (1e-2 * randn(case["rows"], case["cols"])).to(dt)
        s["seed"], s["offset"] = 0x5EED_0123_4567 + seed, 17 * seed + 3
        return s
    if op == "logprobs":
        n, v = case["rows"], case["vocab"]
        s["ids"] = _tokens(gen, n, v, 0.1 if case["train"] and n > 1 else 0.0)
        z = randn(n, v).mul_(2.0)
        at = s["ids"].clamp(min=0)[:, None]
        # the token that followed is mostly among the likely ones
        z.scatter_add_(1, at, 2.0 + 5.0 * randn(n, 1).abs())
        if case["masked"]:
            out = torch.rand(n, v, generator=gen, device="cuda") < 0.9
            out.scatter_(1, at, False)
            z.masked_fill_(out, -math.inf)
        s["logits"] = z.to(_DTYPES[case["dtype"]])
        if case["train"]:
            s["dlogprob"], s["dentropy"] = _upstream(gen, n)
        return s
    n, w, v = case["tokens"], case["width"], case["vocab"]
    s["ids"] = _tokens(gen, n, v, 0.1 if case["train"] else 0.0)
    x = randn(n, w) * torch.exp(0.2 * randn(w))
    s["x"] = (x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6)).to(torch.bfloat16)
    s["weight"] = randn(v, w).mul_(2.0 * w ** -0.5).to(torch.bfloat16)
    if case["train"]:
        s["dlogprob"], s["dentropy"] = _upstream(gen, n)
    return s


# ------------------------------------------------------------------------ the plain form
def _embed(s):
    ids, w = s["ids"], s["weight"]
    on = (ids >= 0)[:, None]
    rows = w[ids.clamp(min=0)].float() * s["scale"]
    y = torch.where(on, rows, 0.0).to(torch.bfloat16)
    if not s["train"]:
        return y
    g = torch.zeros(s["vocab"], s["width"], device="cuda")
    g.index_add_(0, ids.clamp(min=0), torch.where(on, s["dy"].float(), 0.0))
    return {"y": y, "dtable": (g * s["scale"]).to(w.dtype)}


def _philox(blocks, seed, offset):
    """Eight 16-bit pieces for each of `blocks` counters, whole numbers in int64."""
    low = 0xFFFFFFFF
    c = [blocks & low, blocks >> 32, torch.full_like(blocks, offset & low),
         torch.full_like(blocks, (offset >> 32) & low)]
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57   # 64 bits, the sign bit one of them
        c = [(b >> 32) & low ^ c[1] ^ k0, b & low, (a >> 32) & low ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], 1)


def _dropout(s):
    x = s["x"]
    n = x.numel()
    pieces = _philox(torch.arange(-(-n // 8), device="cuda"), s["seed"], s["offset"])
    least = round(65536 * s["p"])
    keep = (pieces.flatten()[:n] >= least).view_as(x)
    scale = 65536 / (65536 - least)
    y = torch.where(keep, x.float() * scale, 0.0)
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": y.to(x.dtype), "dx": torch.where(keep, s["dy"].float() * scale, 0.0).to(x.dtype)}


def _statistics(z, ids):
    """The log of the sum of exponentials, the entropy and the tokens' log probabilities."""
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    p = e / total
    entropy = -torch.where(p > 0, p * (z - lse), 0.0).sum(1)
    taken = z.gather(1, ids.clamp(min=0)[:, None])[:, 0]
    lse = lse[:, 0]
    return lse, entropy, torch.where(ids >= 0, taken - lse, 0.0)


def _score_gradient(z, ids, lse, entropy, dlogprob, dentropy):
    d = z - lse[:, None]
    p = torch.exp(d)
    g = torch.where(ids >= 0, dlogprob, 0.0)[:, None]
    dz = -g * p - torch.where(p > 0, dentropy[:, None] * p * (d + entropy[:, None]), 0.0)
    return dz.scatter_add_(1, ids.clamp(min=0)[:, None], g)


def _logprobs(s):
    z = s["logits"].float()
    lse, entropy, logprob = _statistics(z, s["ids"])
    out = {"logprob": logprob, "entropy": entropy, "lse": lse}
    if s["top"]:
        v, at = torch.sort(z, dim=1, descending=True, stable=True)
        out["top_logprobs"] = v[:, :s["top"]] - lse[:, None]
        out["top_tokens"] = at[:, :s["top"]]
    if s["train"]:
        out["dlogits"] = _score_gradient(z, s["ids"], lse, entropy, s["dlogprob"],
                                         s["dentropy"]).to(s["logits"].dtype)
    return out


def _head(s):
    x, w = s["x"].float(), s["weight"].float()
    z = x @ w.t()
    lse, entropy, logprob = _statistics(z, s["ids"])
    out = {"logprob": logprob, "entropy": entropy, "lse": lse}
    if s["train"]:
        dz = _score_gradient(z, s["ids"], lse, entropy, s["dlogprob"], s["dentropy"])
        out["dx"] = (dz @ w).to(torch.bfloat16)
        out["dweight"] = (dz.t() @ x).to(torch.bfloat16)
    return out


# ------------------------------------------------------------------------ the calls
def _own(s):
    import paper_2606_13894_amd as gf
    op = s["op"]
    if op == "embed":
        y = gf.embedding(s["ids"], s["weight"], scale=s["scale"], dtype=torch.bfloat16)
        if not s["train"]:
            return y
        return {"y": y, "dtable": gf.embedding_backward(s["dy"], s["ids"], s["vocab"],
                                                        scale=s["scale"],
                                                        dtype=s["weight"].dtype)}
    if op == "dropout":
        return {"y": gf.dropout(s["x"], s["p"], s["seed"], s["offset"], residual=s["r"]),
                "dx": gf.dropout(s["dy"], s["p"], s["seed"], s["offset"])}
    if op == "logprobs":
        r = gf.token_logprobs(s["logits"], s["ids"], top=s["top"])
        out = {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse}
        if s["top"]:
            out["top_logprobs"], out["top_tokens"] = r.top_logprobs, r.top_tokens
        if s["train"]:
            out["dlogits"] = gf.token_logprobs_backward(
                s["dlogprob"], s["logits"], s["ids"], r.lse, r.entropy, dentropy=s["dentropy"])
        return out
    r = gf.head_logprobs(s["x"], s["weight"], s["ids"])
    out = {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse}
    if s["train"]:
        out["dx"], out["dweight"] = gf.head_logprobs_backward(
            s["dlogprob"], s["x"], s["weight"], s["ids"], r.lse, r.entropy,
            dentropy=s["dentropy"])
    return out


def run(state):
    if own:
        return _own(state)
    return {"embed": _embed, "dropout": _dropout, "logprobs": _logprobs,
            "head": _head}[state["op"]](state)


# ------------------------------------------------------------------------ 64 bits
def _pieces64(n, seed, offset):
    """The same 16-bit pieces in numpy's 64-bit unsigned numbers."""
    low = np.uint64(0xFFFFFFFF)
    i = np.arange((n + 7) // 8, dtype=np.uint64)
    x0, x1 = i & low, i >> np.uint64(32)
    x2, x3 = np.full_like(i, offset % 2 ** 32), np.full_like(i, offset // 2 ** 32 % 2 ** 32)
    for r in range(10):
        key = [np.uint64((seed // 2 ** (32 * j) + r * w) % 2 ** 32)
               for j, w in enumerate((0x9E3779B9, 0xBB67AE85))]
        first, second = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1 = (second >> np.uint64(32)) ^ x1 ^ key[0], second & low
        x2, x3 = (first >> np.uint64(32)) ^ x3 ^ key[1], first & low
    words = np.stack([x0, x1, x2, x3], 1).astype("<u4")
    return words.reshape(-1).view("<u2")[:n].astype(np.int64)


def _head64(z, s):
    """Everything that is asked of float64 logits, the rows in pieces that fit beside them."""
    ids = s["ids"]
    n = z.shape[0]
    lse, entropy, logprob = (torch.empty(n, device="cuda", dtype=torch.float64) for _ in range(3))
    dz = torch.empty_like(z) if s["train"] else None
    for a in range(0, n, 512):
        rows = slice(a, min(n, a + 512))
        zr, t = z[rows], ids[rows]
        lse[rows] = torch.logsumexp(zr, 1)
        lp = zr - lse[rows, None]
        p = lp.exp()
        plogp = torch.nan_to_num(p * lp, nan=0.0)     # 0 times the log of 0
        entropy[rows] = -plogp.sum(1)
        on = t >= 0
        hit = torch.zeros_like(zr, dtype=torch.bool)
        hit[on.nonzero()[:, 0], t[on]] = True
        logprob[rows] = torch.where(hit, lp, 0.0).sum(1)
        if dz is not None:
            g = torch.where(on, s["dlogprob"][rows].double(), 0.0)[:, None]
            dz[rows] = g * (hit.double() - p) - s["dentropy"][rows].double()[:, None] * (
                plogp + p * entropy[rows, None])
    return lse, entropy, logprob, dz


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        ids, n = s["ids"], case["tokens"]
        y = torch.zeros(n, case["width"], device="cuda", dtype=torch.float64)
        on = ids >= 0
        y[on] = s["weight"][ids[on]].double() * s["scale"]
        if not case["train"]:
            return y
        order = torch.argsort(ids[on], stable=True)
        at, dy = ids[on][order], s["dy"][on][order].double()
        upto = torch.cat([torch.zeros_like(dy[:1]), dy.cumsum(0)])
        first = torch.searchsorted(at, torch.arange(case["vocab"] + 1, device="cuda"))
        g = torch.zeros(case["vocab"], case["width"], device="cuda", dtype=torch.float64)
        used = (first[1:] > first[:-1]).nonzero()[:, 0]
        g[used] = (upto[first[used + 1]] - upto[first[used]]) * s["scale"]
        return {"y": y, "dtable": g}
    if op == "dropout":
        x = s["x"].double()
        least = round(65536 * case["p"])
        pieces = torch.from_numpy(_pieces64(x.numel(), s["seed"], s["offset"])).to("cuda")
        factor = (pieces >= least).double().view_as(x) * (65536 / (65536 - least))
        y = x * factor
        if s["r"] is not None:
            y = y + s["r"].double()
        return {"y": y, "dx": s["dy"].double() * factor}
    if op == "logprobs":
        z = s["logits"].double()
        lse, entropy, logprob, dz = _head64(z, s)
        out = {"logprob": logprob, "entropy": entropy}
        if case["top"]:
            best, where = [], []
            left = z.clone()
            for _ in range(case["top"]):
                m = left.amax(1, keepdim=True)
                column = torch.arange(z.shape[1], device="cuda").expand_as(left)
                at = torch.where(left == m, column, z.shape[1]).amin(1, keepdim=True)
                best.append(m - lse[:, None])
                where.append(at)
                left.scatter_(1, at, -math.inf)
            out["top_logprobs"], out["top_tokens"] = torch.cat(best, 1), torch.cat(where, 1)
        if case["train"]:
            out["dlogits"] = dz
        return out
    x, w = s["x"].double(), s["weight"].double()
    lse, entropy, logprob, dz = _head64(torch.mm(x, w.t()), s)
    out = {"logprob": logprob, "entropy": entropy, "lse": lse}
    if case["train"]:
        out["dx"], out["dweight"] = torch.mm(dz, w), torch.mm(dz.t(), x)
    return out


# ------------------------------------------------------------------------ what a pass needs
def work(case):
    op = case["op"]
    if op == "embed":
        n, v, w = case["tokens"], case["vocab"], case["width"]
        size = 4 if case["table"] == "f32" else 2
        rows = min(n, v) if case["train"] else n          # rows of the table that are read
        forward = 8 * n + rows * w * size + 2 * n * w
        back = 8 * n + 2 * n * w + v * w * size
        return {"bytes": forward + (back if case["train"] else 0),
                "flops": n * w * (3 if case["train"] else 1)}
    if op == "dropout":
        n = case["rows"] * case["cols"]
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": n * size * (5 if case["residual"] else 4), "flops": 4 * n}
    if op == "logprobs":
        n = case["rows"] * case["vocab"]
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": n * size * (3 if case["train"] else 1)
                + case["rows"] * (16 + 12 * case["top"]),
                "flops": n * (14 if case["train"] else 6)}
    t, w, v = case["tokens"], case["width"], case["vocab"]
    one = 2 * v * w + 2 * t * w + 16 * t
    return {"bytes": one * (3 if case["train"] else 1),
            "flops": 2 * t * w * v * (3 if case["train"] else 1)}
