"""Speculative decode steps around a vocabulary table held in 4 bits.

One table serves the head, the next step's inputs and a training step of its own:

  quantise    the table's rows into 4 bits, once
  lookup      the inputs of the step's rows from their tokens
  product     target logits over a language subset, hidden states in 3 terms
  verify      the drafts against them (sph_verify_draft, on the same context)
  gradient    of the table, from the gradients of the rows that were looked up

The decoder between inputs and head is another program's; a fixed rotation and an
RMS norm stand in for it here, and greedy drafts from the step before for its draft
module.  Run on a GPU:  python examples/four_bit_step.py
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def run(V=32000, d=1024, sessions=8, k=4, keep_fraction=0.4, steps=3, seed=0):
    """A few steps; returns the accepted counts and next tokens of each, the bytes of
    the table in 4 bits and in bf16, and the table's gradient."""
    from paper_2607_13093_gb300 import sph
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    ctx = sph.Context(dev.index)
    table = (torch.randn(V, d, generator=g, device=dev) * 0.02).to(torch.bfloat16)
    held = ctx.mx4_quantize(table, sph.SPH_MX4_E4M3)
    keep = (torch.rand(V, generator=g, device=dev) < keep_fraction).nonzero()[:, 0].to(torch.int32)
    rows = sessions * (k + 1)
    mix = torch.randn(d, d, generator=g, device=dev) / math.sqrt(d)

    tokens = keep[torch.randint(0, keep.numel(), (rows,), generator=g, device=dev)]
    x = torch.empty(rows, d, device=dev)                     # inputs, fp32
    z = torch.empty(rows, keep.numel(), device=dev)          # target logits
    history, seen = [], []
    for step in range(steps):
        ctx.embed(tokens, held, scale=math.sqrt(d), out=x)
        h = x @ mix
        h = h / h.square().mean(1, keepdim=True).sqrt()
        ctx.mx4_logits(h, held, keep_ids=keep, planes=3, out=z)
        drafts = tokens.view(sessions, k + 1)[:, 1:].contiguous()
        accepted, next_token = ctx.verify_draft(z, sessions, k, drafts, keep_ids=keep,
                                                temperature=0.8, seed=seed, offset=step)
        history.append((accepted, next_token))
        seen.append(tokens)
        # the next step's rows: the token just drawn, then greedy drafts
        best = keep[z.view(sessions, k + 1, -1)[:, :k].argmax(2)]
        tokens = torch.cat([next_token[:, None], best], 1).reshape(-1).contiguous()
    # training: the table's gradient from the gradients of the inputs, summed over the
    # occurrences of a token; the second call adds to the first
    grad = torch.empty(V, d, device=dev)
    for i, t in enumerate(seen):
        d_x = torch.randn(rows, d, generator=g, device=dev) * 1e-2
        ctx.embed_grad(t, d_x, V, scale=math.sqrt(d), out=grad, accumulate=i > 0)
    ctx.sync()
    bits4 = sum(t.numel() * t.element_size() for t in held[:3] if t is not None)
    ctx.close()
    return dict(history=history, keep=keep, bits4=bits4, bf16=table.numel() * 2, grad=grad, seen=seen)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--dim", type=int, default=1024)
    ap.add_argument("--sessions", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--steps", type=int, default=3)
    a = ap.parse_args()
    r = run(a.vocab, a.dim, a.sessions, a.drafts, steps=a.steps)
    print(f"table: {r['bf16'] / 1e6:.1f} MB in bf16, {r['bits4'] / 1e6:.1f} MB in 4 bits")
    for i, (n, t) in enumerate(r["history"]):
        print(f"step {i}: accepted {n.tolist()} next {t.tolist()}")
    print(f"gradient: {int((r['grad'] != 0).any(1).sum())} rows of {a.vocab} touched")


if __name__ == "__main__":
    main()
