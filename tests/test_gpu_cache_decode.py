"""-m gpu: examples/beam_decode.py with norms, tokens that all sources have in common, and a budget for the sources, against the same decoder without a cache.

Tolerance: as in test_gpu_beam_decode.py; norms keep scores' sizes.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_beam_decode import TOLERANCE, example, rotated  # noqa: F401

pytestmark = pytest.mark.gpu


def log_probs(dec, ids):
    """[n, V] in 64 bits on the CPU: the whole sequence at once, no cache."""
    w = {n: [t.double().cpu() for t in getattr(dec, n)] for n in ("qkv", "out", "remember")}
    norm = lambda x: x / x.norm(dim=-1, keepdim=True) * x.shape[-1] ** 0.5
    x, n, D = dec.embed.double().cpu()[torch.tensor(ids)], len(ids), dec.head_dim
    inv = dec.inv_freq.double().cpu()
    for layer in range(dec.layers):
        y = (norm(x) @ w["qkv"][layer]).unflatten(-1, (dec.q_heads + 2 * dec.heads, D))
        q, k, v = y[:, :dec.q_heads], y[:, dec.q_heads:-dec.heads], y[:, -dec.heads:]
        if dec.norms[layer]:
            by_head = lambda x, weight: x / (x.square().mean(dim=-1, keepdim=True) + 1e-6).sqrt() * dec.norms[layer][weight].double().cpu()
            q, k = by_head(q, "q_weight"), by_head(k, "k_weight")
        q, k = rotated(q, inv), rotated(k, inv)
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


@pytest.mark.parametrize("P,norms,budget", [(0, True, None), (21, False, None), (21, True, None), (21, True, 23), (0, False, 30)])
def test_scores_of_a_decode(example, P, norms, budget):  # noqa: F811
    """A budget that leaves every source whole moves it, and changes nothing."""
    B, S, k, V, steps = 3, 23, 4, 60, 14
    g = torch.Generator().manual_seed(5)
    dec = example.Decoder(V, layers=2, q_heads=4, heads=2, head_dim=32, dtype=torch.float32, norms=norms)
    dec.to_logits[:, example.EOS] += 0.02
    source, lengths = torch.randint(3, V, (B, S), generator=g), torch.tensor([23, 1, 9])
    common = torch.randint(3, V, (P,), generator=g) if P else None
    with torch.no_grad():
        tokens, backs, score, flags = example.decode(dec, source.cuda(), lengths, k, steps, page=8, common=common, budget=budget)
    for b in range(B):
        alive = [h for h in range(k) if not flags[b, h] & 2]
        assert alive and len({tuple(example.path(tokens, backs, b, h)) for h in alive}) == len(alive)
        for h in alive:
            out = example.path(tokens, backs, b, h)
            src = (common.tolist() if P else []) + source[b, :int(lengths[b])].tolist()
            lp = log_probs(dec, src + out[:-1])
            want = 0.0
            for i, w in enumerate(out):
                want += float(lp[len(src) - 1 + i, w])
                if w == example.EOS:
                    break
            assert abs(score[b, h] - want) <= TOLERANCE, (b, h, score[b, h], want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_a_decode_with_a_budget_ends_with_a_full_beam(example, dtype):  # noqa: F811
    B, S, k, V, steps = 4, 40, 6, 700, 20
    dec = example.Decoder(V, dtype=dtype, norms=True)
    g = torch.Generator().manual_seed(2)
    source, common = torch.randint(3, V, (B, S), generator=g).cuda(), torch.randint(3, V, (70,), generator=g)
    with torch.no_grad():
        tokens, backs, score, flags = example.decode(dec, source, torch.tensor([40, 3, 17, 33]), k, steps, common=common, budget=10)
    assert np.isfinite(score).all() and not (flags & 2).any() and (np.diff(score, axis=1) <= 0).all()
