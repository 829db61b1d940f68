"""Train a small model of tokens with Gefen, from the embedding table to the log probabilities, and
score single tokens with it.

    python examples/train_tokens.py [--vocab 4096] [--layers 2] [--width 256] [--steps 100]

Tokens become rows of the embedding table (``Embedding``), a share of them is dropped (``Dropout``, whose
mask is never stored), feed-forward blocks follow (``FeedForward``), and the output head gives the
log probability of each next token without storing a score (``Head``). The head's weight is the
table itself with ``--tied``. There is no attention: the text is synthetic and each token depends on the
one before it alone, the first third of each sequence is a prompt that no loss is taken on.
Prints the loss, the time of a step and what the scores would have taken; then the log probabilities and
best alternatives of a few single tokens.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_13894_amd as gf  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, vocab, width, inner, layers, dropout, tied, device):
        super().__init__()
        self.embed = gf.Embedding(vocab, width, scale=width ** 0.5, device=device)
        self.drop = gf.Dropout(dropout, seed=1, device=device)
        self.blocks = torch.nn.ModuleList(
            gf.FeedForward(width, inner, device=device, dropout=dropout, seed=2 + i)
            for i in range(layers))
        self.norm = torch.nn.Parameter(torch.ones(width, device=device))
        self.head = gf.Head(width, vocab, weight=self.embed.table if tied else None, device=device)

    def forward(self, tokens, following):
        """The log probability of each following token, and the entropy there."""
        y, h = self.drop(self.embed(tokens)), None
        for block in self.blocks:
            y, h = block(y, h)
        x = y + h
        # (torch's norm: the library's plain call has no gradient of its own)
        x = torch.nn.functional.rms_norm(x.float(), x.shape[-1:], self.norm, 1e-6)
        return self.head(x.to(torch.bfloat16), following)


def scorer(model):
    """Single tokens without autograd: the weights are cast once, nothing is saved."""
    bf16 = torch.bfloat16
    table = model.embed.table.detach().to(bf16)
    head = model.head.weight.detach().to(bf16)
    blocks = [(b.norm.detach(), b.w_gate.detach().to(bf16), b.w_up.detach().to(bf16),
               b.w_down.detach().to(bf16), b.eps, b.activation) for b in model.blocks]

    def hidden(tokens):
        y, h = gf.embedding(tokens, table, scale=model.embed.scale), None
        for norm, wg, wu, wd, eps, act in blocks:
            n = gf.rms_norm(y, norm, residual=h, eps=eps)
            y, h = gf.gated_ffn(n.y, wg, wu, wd, activation=act), n.h
        return gf.rms_norm(y, model.norm.detach(), residual=h).y

    def score(tokens, following, top):
        """From the head without scores, and from the scores themselves with alternatives."""
        x = hidden(tokens)
        taken = gf.head_logprobs(x, head, following)
        return taken, gf.token_logprobs(x @ head.t(), following, top=top)

    return score


def text(follow, sequences, length, device):
    """Tokens whose next one is one of four that the token decides."""
    t = torch.randint(follow.shape[0], (sequences,), device=device)
    out = [t]
    for _ in range(length):
        t = follow[t, torch.randint(follow.shape[1], (sequences,), device=device)]
        out.append(t)
    return torch.stack(out, 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--inner", type=int, default=1024)
    ap.add_argument("--sequences", type=int, default=16)
    ap.add_argument("--length", type=int, default=256)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--lr", type=float, default=1e-3)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--tied", action="store_true")
    a = ap.parse_args(argv)
    dev = torch.device("cuda", torch.cuda.current_device())
    torch.manual_seed(0)
    model = Model(a.vocab, a.width, a.inner, a.layers, a.dropout, a.tied, dev)
    follow = torch.randint(a.vocab, (a.vocab, 4), device=dev)
    opt = gf.Gefen(model.parameters(), lr=a.lr, weight_decay=0.0)
    first = last = begin = 0.0
    for step in range(a.steps):
        t = text(follow, a.sequences, a.length, dev)
        tokens, following = t[:, :-1], t[:, 1:].clone()
        following[:, :a.length // 3] = -1                  # the prompt
        logprob, _ = model(tokens, following)
        loss = -logprob.sum() / (following >= 0).sum()
        opt.zero_grad()
        loss.backward()
        opt.step()
        if step == 0:
            first = last = loss.item()
            begin = time.perf_counter()
        elif step + 1 == a.steps or step % 20 == 0:
            last = loss.item()
            print(f"step {step}: loss {last:.4f} (first {first:.4f})", flush=True)
    torch.cuda.synchronize()
    ms = 1e3 * (time.perf_counter() - begin) / max(1, a.steps - 1)
    scores = 4 * a.sequences * a.length * a.vocab / 2**20
    print(f"{ms:.2f} ms a step; the scores, never stored, would be {scores:.0f} MiB in float32")
    model.eval()
    score = scorer(model)
    tokens = torch.arange(3, device=dev)
    following = follow[tokens, 0]
    taken, best = score(tokens, following, 4)
    # the scores there are rounded to bfloat16, here they are not
    off = (taken.logprob - best.logprob).abs().max().item()
    for i in range(3):
        print(f"token {i}: next {following[i].item()} has log probability "
              f"{taken.logprob[i].item():.3f}, entropy {taken.entropy[i].item():.3f}; best "
              f"{best.top_tokens[i].tolist()} of {follow[i].tolist()}")
    return first, last, off


if __name__ == "__main__":
    main()
