#!/usr/bin/env python3
"""Beam search with a small attention decoder around the operators of include/dba_beam.h.

The decoder is a stand-in with random weights (attention over a paged cache with rotated keys, a gated recurrent memory
beside it); its products are torch's, what the search does around them is the library's:

    append    the time step's keys and values go into the cache, one token for every slot of the beam
    attend    every slot attends over the source and its own ancestors among the generated tokens (a row of mask bits)
    select    the new beam from the logits; with --constraints dba_step chooses instead, from log-probs
    reorder   mask rows and the recurrent memories follow the back-pointers; keys and values stay where they are

    python examples/beam_decode.py [--batch 4] [--beam 5] [--vocab 8000] [--steps 24] [--dtype bf16] [--constraints]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

PAD, EOS = 0, 2
FINISHED, DEAD = 1, 2


class Decoder:
    """Weights of `layers` blocks of grouped-query attention and a recurrent memory, random."""

    def __init__(self, vocab, layers=2, q_heads=8, heads=2, head_dim=64, dtype=torch.bfloat16, device="cuda", seed=1):
        self.vocab, self.layers, self.q_heads, self.heads, self.head_dim = vocab, layers, q_heads, heads, head_dim
        self.dim = q_heads * head_dim
        g = torch.Generator().manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g) * rows ** -0.5).to(dtype).to(device)

        self.embed = torch.randn(vocab, self.dim, generator=g).to(dtype).to(device)
        self.qkv = [weight(self.dim, (q_heads + 2 * heads) * head_dim) for _ in range(layers)]
        self.out = [weight(self.dim, self.dim) for _ in range(layers)]
        self.remember = [weight(self.dim, 2 * self.dim) for _ in range(layers)]
        self.to_logits = weight(self.dim, vocab) * 2
        self.inv_freq = (10000.0 ** (-torch.arange(0, head_dim, 2).double() / head_dim)).float().to(device)

    @staticmethod
    def norm(x):
        return torch.nn.functional.normalize(x.float(), dim=-1).mul(x.shape[-1] ** 0.5).to(x.dtype)

    def split(self, layer, x):
        """x [B, n, dim] -> q, k, v [B, n, heads, head_dim], views of one product."""
        y = torch.matmul(self.norm(x), self.qkv[layer]).unflatten(-1, (self.q_heads + 2 * self.heads, self.head_dim))
        return y[:, :, :self.q_heads], y[:, :, self.q_heads:-self.heads], y[:, :, -self.heads:]

    def update(self, layer, x, memory):
        """One step of the recurrent memory [.., dim] (fp32): (x with it, the new one)."""
        gate, new = torch.matmul(self.norm(x), self.remember[layer]).float().chunk(2, dim=-1)
        gate = gate.sigmoid()
        memory = memory * gate + (1 - gate) * new
        return x + memory.to(x.dtype), memory

    def logits(self, x):
        return torch.matmul(self.norm(x), self.to_logits)


def decode(dec, source, lengths, k, steps, page=16, constraints=None):
    """Beam search behind the sources [B, S] (the first lengths[b] tokens of each).  Returns tokens, back-pointers, each [steps, B, k], and
    the last beam's scores and flags [B, k], on the host.  constraints: the CSR arrays of dba_init."""
    from paper_1804_06609_amd import beam
    from paper_1804_06609_amd.session import Session

    dev = source.device
    B, S = source.shape
    dtype, heads, D, L = dec.embed.dtype, dec.heads, dec.head_dim, dec.layers
    # one table of pages for all layers' pools, pages in any order
    per = -(-(S + k * steps) // page)
    table = torch.randperm(B * per, device=dev).to(torch.int32).reshape(B, per)
    pools = [[torch.empty((B * per, page, heads, D), dtype=dtype, device=dev) for _ in range(2)] for _ in range(L)]
    lens = lengths.to(torch.int32).to(dev)
    start, whole = torch.zeros_like(lens), torch.full_like(lens, S)

    # the sources: a chain of tokens each
    x = dec.embed[source]
    memory = []
    last = (lens.long() - 1)[:, None, None].expand(B, 1, dec.dim)
    for layer in range(L):
        q, key, value = dec.split(layer, x)
        q = beam.append(key, value, *pools[layer], table, start, lens, inv_freq=dec.inv_freq, q=q)
        o = beam.attend(q, *pools[layer], table, start, whole, max_len=S)
        x = x + torch.matmul(o.flatten(2), dec.out[layer])
        m, ys = torch.zeros(B, dec.dim, device=dev), []
        for t in range(S):
            y, new = dec.update(layer, x[:, t], m)
            m = torch.where((t < lens)[:, None], new, m)
            ys.append(y)
        x = torch.stack(ys, dim=1)
        memory.append(m[:, None].expand(B, k, dec.dim).contiguous())
    logits = dec.logits(x.gather(1, last))                              # [B, 1, V]

    words = -(-k * steps // 64)
    mask = torch.zeros((B, k, words), dtype=torch.int64, device=dev)    # bit t * k + h: the token of slot h at step t
    slots = torch.arange(k, device=dev)
    score, flags = torch.zeros((B, 1), device=dev), None
    ses = None
    if constraints is not None:
        ses = Session(B, k, dec.vocab, steps, EOS, PAD, *constraints)
        logits = logits.expand(B, k, dec.vocab)                         # (before the first step only slot 0 is live)
    tokens, backs = [], []
    try:
        for t in range(steps):
            if ses is not None:
                ses.step(torch.log_softmax(logits.float(), dim=2))
                token, back, score, flags = (o.clone() for o in (ses.out_token, ses.out_backptr, ses.out_score, ses.out_flags))
            else:
                token, back, score, flags = beam.select(logits.contiguous(), score, flags, k, EOS, PAD)
            tokens.append(token)
            backs.append(back)
            if t + 1 == steps:
                break
            if t:                                                       # (the slots of the first beam all come from the source)
                beam.reorder(back, [mask] + memory)
            bit = t * k + slots
            mask |= torch.where(torch.arange(words, device=dev)[None] == (bit >> 6)[:, None], (torch.ones_like(bit) << (bit & 63))[:, None], 0)[None]
            first, tree = lens + t * k, torch.full_like(lens, (t + 1) * k)
            depth = (lens + t)[:, None].expand(B, k).contiguous()       # the beam's tokens stand side by side in the cache, all at one position
            x = dec.embed[token.long()]
            for layer in range(L):
                q, key, value = dec.split(layer, x)
                q = beam.append(key, value, *pools[layer], table, first, position=depth, inv_freq=dec.inv_freq, q=q)
                o = beam.attend(q, *pools[layer], table, lens, tree, mask, max_len=S + (t + 1) * k)
                x = x + torch.matmul(o.flatten(2), dec.out[layer])
                x, memory[layer] = dec.update(layer, x, memory[layer])
            logits = dec.logits(x)
        return tuple(y.cpu().numpy() for y in (torch.stack(tokens), torch.stack(backs), score, flags))
    finally:
        if ses is not None:
            ses.close()


def path(tokens, backs, b, h):
    """The tokens of slot h of the last beam, first to last."""
    out = []
    for t in range(len(tokens) - 1, -1, -1):
        out.append(int(tokens[t, b, h]))
        h = int(backs[t, b, h])
    return out[::-1]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--beam", type=int, default=5)
    ap.add_argument("--vocab", type=int, default=8000)
    ap.add_argument("--source", type=int, default=30)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--dtype", choices=("f32", "f16", "bf16"), default="bf16")
    ap.add_argument("--constraints", action="store_true", help="two tokens that every sentence has to contain")
    args = ap.parse_args()
    dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[args.dtype]
    g = torch.Generator().manual_seed(3)
    source = torch.randint(3, args.vocab, (args.batch, args.source), generator=g).cuda()
    lengths = torch.randint(1, args.source + 1, (args.batch,), generator=g)
    constraints = None
    if args.constraints:
        wanted = torch.randint(3, args.vocab, (2 * args.batch,), generator=g).int().numpy()
        constraints = wanted, np.arange(2 * args.batch + 1, dtype=np.int32), np.arange(0, 2 * args.batch + 1, 2, dtype=np.int32)
    with torch.no_grad():
        tokens, backs, score, flags = decode(Decoder(args.vocab, dtype=dtype), source, lengths, args.beam, args.steps, constraints=constraints)
    for b in range(args.batch):
        live = [h for h in range(args.beam) if not flags[b, h] & DEAD]
        print(f"sentence {b}: {len(live)} hypotheses, best {score[b, live[0]]:.3f}: {' '.join(map(str, path(tokens, backs, b, live[0])))}")


if __name__ == "__main__":
    main()
