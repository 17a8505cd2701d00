"""-m gpu: examples/beam_decode.py - the operators of include/dba_beam.h run together - against the same decoder without a cache.

Tolerance: a score is the sum of at most 14 log-probs of logits around 2 in size; each is the end of two layers of fp32 products of at
most 512 terms (2^-24 * 512 = 3e-5 of themselves at worst), so 14 * 2 * 3e-5 < 1e-3.
"""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOLERANCE = 1e-3


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("beam_decode", os.path.join(ROOT, "examples", "beam_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def rotated(x, inv_freq):
    """x [n, heads, D] at positions 0 .. n-1, in 64 bits."""
    angle = torch.arange(len(x)).double()[:, None] * inv_freq[None]
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x.chunk(2, dim=-1)
    return torch.cat((a * c - b * s, b * c + a * s), dim=-1)


def log_probs(dec, ids):
    """[n, V] in 64 bits on the CPU: the whole sequence at once, no cache."""
    w = {n: [t.double().cpu() for t in getattr(dec, n)] for n in ("qkv", "out", "remember")}
    norm = lambda x: x / x.norm(dim=-1, keepdim=True) * x.shape[-1] ** 0.5
    x, n, D = dec.embed.double().cpu()[torch.tensor(ids)], len(ids), dec.head_dim
    inv = dec.inv_freq.double().cpu()
    for layer in range(dec.layers):
        y = (norm(x) @ w["qkv"][layer]).unflatten(-1, (dec.q_heads + 2 * dec.heads, D))
        q, k, v = rotated(y[:, :dec.q_heads], inv), rotated(y[:, dec.q_heads:-dec.heads], inv), y[:, -dec.heads:]
        k, v = (t.repeat_interleave(dec.q_heads // dec.heads, dim=1) for t in (k, v))
        s = torch.stack([q[:, h] @ k[:, h].T for h in range(dec.q_heads)]) / math.sqrt(D)
        p = s.masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf).softmax(dim=2)
        x = x + torch.stack([p[h] @ v[:, h] for h in range(dec.q_heads)], dim=1).flatten(1) @ w["out"][layer]
        memory, rows = torch.zeros(dec.dim).double(), []
        for t in range(n):
            gate, new = (norm(x[t]) @ w["remember"][layer]).chunk(2)
            memory = memory * gate.sigmoid() + (1 - gate.sigmoid()) * new
            rows.append(x[t] + memory)
        x = torch.stack(rows)
    return torch.log_softmax(norm(x) @ dec.to_logits.double().cpu(), dim=1)


def check_scores(example, dec, source, lengths, tokens, backs, score, flags):
    B, k = score.shape
    for b in range(B):
        alive = [h for h in range(k) if not flags[b, h] & 2]
        assert alive and len({tuple(example.path(tokens, backs, b, h)) for h in alive}) == len(alive)
        assert (np.diff(score[b, alive]) <= 0).all()
        for h in alive:
            out = example.path(tokens, backs, b, h)
            src = source[b, :int(lengths[b])].tolist()
            lp = log_probs(dec, src + out[:-1])
            want = 0.0
            for i, w in enumerate(out):
                want += float(lp[len(src) - 1 + i, w])
                if w == example.EOS:
                    assert all(y == example.PAD for y in out[i + 1:]) and flags[b, h] & 1
                    break
            assert abs(score[b, h] - want) <= TOLERANCE, (b, h, score[b, h], want)


@pytest.mark.parametrize("constrained", [False, True])
def test_scores_of_a_decode(example, constrained):
    B, S, k, V, steps = 3, 23, 4, 60, 14
    g = torch.Generator().manual_seed(5)
    dec = example.Decoder(V, layers=2, q_heads=4, heads=2, head_dim=32, dtype=torch.float32)
    dec.to_logits[:, example.EOS] += 0.02                                # (some hypotheses complete)
    source, lengths = torch.randint(3, V, (B, S), generator=g), torch.tensor([23, 1, 9])
    wanted = torch.randint(3, V, (2 * B,), generator=g).int().numpy()
    constraints = (wanted, np.arange(2 * B + 1, dtype=np.int32), np.arange(0, 2 * B + 1, 2, dtype=np.int32)) if constrained else None
    with torch.no_grad():
        got = example.decode(dec, source.cuda(), lengths, k, steps, page=8, constraints=constraints)
    check_scores(example, dec, source, lengths, *got)
    if constrained:
        tokens, backs, score, flags = got
        for b in range(B):
            assert any({int(wanted[2 * b]), int(wanted[2 * b + 1])} <= set(example.path(tokens, backs, b, h)) for h in range(k) if not flags[b, h] & 2)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_decode_in_16_bits_ends_with_a_full_beam(example, dtype):
    B, S, k, V, steps = 4, 40, 6, 700, 20
    dec = example.Decoder(V, dtype=dtype)
    source = torch.randint(3, V, (B, S), generator=torch.Generator().manual_seed(2)).cuda()
    with torch.no_grad():
        tokens, backs, score, flags = example.decode(dec, source, torch.tensor([40, 3, 17, 33]), k, steps)
    assert np.isfinite(score).all() and not (flags & 2).any() and (np.diff(score, axis=1) <= 0).all()
