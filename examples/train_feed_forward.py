"""Train a stack of feed-forward blocks with Gefen: one byte per saved activation, one byte of
optimizer state per weight.

    python examples/train_feed_forward.py [--layers 4] [--width 512] [--inner 2048] [--steps 100]

Each block is h = x + residual, y = its gated block of the RMS norm of h (``FeedForward``); y and h
go on as the next block's x and residual, so that the residual's addition is always the norm
kernel's. The task is synthetic: a random teacher of the same shape to be matched. After training
the stack answers single tokens without saving anything. Prints the loss, the time of a step, and
the bytes of activations kept for the backward pass beside those of a bfloat16 implementation (h,
its norm, both projections and their product), and those of the bfloat16 weights kept with them.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_13894_amd as gf  # noqa: E402


class Stack(torch.nn.Module):
    def __init__(self, layers, width, inner, device):
        super().__init__()
        self.blocks = torch.nn.ModuleList(
            gf.FeedForward(width, inner, device=device) for _ in range(layers))

    def forward(self, x):
        y, h = x, None
        for block in self.blocks:
            y, h = block(y, h)
        return y + h


def serve(stack, x):
    """The same stack without autograd: nothing is saved. bfloat16 weights are made once."""
    bf16 = torch.bfloat16
    weights = [(b.norm.detach(), b.w_gate.detach().to(bf16), b.w_up.detach().to(bf16),
                b.w_down.detach().to(bf16), b.eps, b.activation) for b in stack.blocks]

    def answer(x):
        y, h = x, None
        for norm, wg, wu, wd, eps, act in weights:
            n = gf.rms_norm(y, norm, residual=h, eps=eps)
            y, h = gf.gated_ffn(n.y, wg, wu, wd, activation=act), n.h
        return y + h

    return answer


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--inner", type=int, default=2048)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--lr", type=float, default=1e-3)
    a = ap.parse_args(argv)
    dev = torch.device("cuda", torch.cuda.current_device())
    torch.manual_seed(0)
    teacher, stack = (Stack(a.layers, a.width, a.inner, dev) for _ in range(2))
    opt = gf.Gefen(stack.parameters(), lr=a.lr, weight_decay=0.0)
    first = last = 0.0
    kept = []
    begin = 0.0
    for step in range(a.steps):
        x = torch.randn(a.tokens, a.width, device=dev).to(torch.bfloat16)
        with torch.no_grad():
            target = teacher(x).float()
        keep = kept.append if step == 0 else lambda t: None
        with torch.autograd.graph.saved_tensors_hooks(lambda t: (keep(t), t)[1], lambda t: t):
            out = stack(x)
        loss = (out.float() - target).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        if step == 0:
            first = loss.item()
            begin = time.perf_counter()
        elif step + 1 == a.steps or step % 20 == 0:
            last = loss.item()
            print(f"step {step}: loss {last:.4f} (first {first:.4f})", flush=True)
    torch.cuda.synchronize()
    ms = 1e3 * (time.perf_counter() - begin) / max(1, a.steps - 1)
    copies = sum(2 * t.numel() for t in kept if t.dtype is torch.bfloat16)
    saved = sum(t.numel() * t.element_size() for t in kept
                if t.dtype in (torch.int8, torch.uint8) or t.shape == (a.tokens,))
    plain = a.layers * a.tokens * 2 * (2 * a.width + 3 * a.inner)
    print(f"{ms:.2f} ms a step; kept for the backward pass: {saved / 2**20:.1f} MiB "
          f"(bfloat16: {plain / 2**20:.1f} MiB), and {copies / 2**20:.1f} MiB of weights")
    answer = serve(stack, x)
    one = answer(x[:1])
    same = stack(x[:1]).detach()   # with gradients: the kernels that save
    err = (one.float() - same.float()).norm() / same.float().norm()
    print(f"one token served: {tuple(one.shape)}, {err:.1e} off the training path")
    return first, last, err.item()


if __name__ == "__main__":
    main()
