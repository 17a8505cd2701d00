"""Workloads by which the speed of the operators around a decoder's paged cache is measured.

A decoder that keeps its keys and values in pages, and whose hypotheses are branches of a tree of cached tokens, does four things more
once its prompts get long: it norms queries and keys by head before it rotates them, by positions of one axis or of several (`append`); it
attends over a prefix that the whole batch has in common and then over each sentence's own tokens (`shared`); it adds up how much
attention each cached token has had (`weigh`); and it keeps of a long cache those that had the most (`evict`).  Ancestor masks come from a search
that was played through, pages lie in the pool in random order, attention weights are heavy-tailed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

ELEM = {"f32": 4, "f16": 2, "bf16": 2}
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def _append(B, n, Hq, Hkv, D, rot, page, lo, hi, dtype, norm, axes=1, prompt=False, interleaved=False):
    """n tokens a sentence behind lo..hi cached ones; prompt: ragged counts from the cache's start.  norm "all": one weight for all heads, "head":
    one for each, "none".  axes: 1, or 3 (time, height, width), whose pairs take turns."""
    return {"op": "append", "B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot, "page": page, "lo": lo, "hi": hi,
            "dtype": dtype, "norm": norm, "axes": axes, "prompt": prompt, "interleaved": interleaved}


def _shared(B, n, Hq, Hkv, D, page, common, lo, hi, steps, dtype, kind):
    """`common` tokens that all sentences have, then lo..hi of their own; kind "beam": behind them `steps` tokens for each of n beam slots, a query
    a slot; "chain": n tokens in a row, all asking."""
    return {"op": "shared", "B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "common": common, "lo": lo, "hi": hi, "steps": steps,
            "dtype": dtype, "kind": kind}


def _weigh(B, n, Hq, Hkv, D, page, lo, hi, steps, dtype, kind, by_head):
    """The same without what is in common; by_head: a score for each head of the cache, else one for all."""
    return {"op": "weigh", "B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "lo": lo, "hi": hi, "steps": steps,
            "dtype": dtype, "kind": kind, "by_head": by_head}


def _evict(B, Hkv, D, page, lo, hi, tree, keep, sinks, recent, dtype, by_head):
    """Of lo..hi tokens a sentence `keep` stay, and the `tree` ones behind them."""
    return {"op": "evict", "B": B, "Hkv": Hkv, "D": D, "page": page, "lo": lo, "hi": hi, "tree": tree, "keep": keep, "sinks": sinks,
            "recent": recent, "dtype": dtype, "by_head": by_head}


def listed():
    return [
        # one hypothesis' next token: launches and latencies only
        dict(_append(1, 1, 8, 8, 64, 64, 16, 1000, 1000, "f32", "all"), name="append_one_token"),
        # a time step of the headline batch, 20 new tokens a sentence
        dict(_append(64, 20, 32, 8, 128, 128, 16, 300, 1500, "bf16", "all"), name="append_beam"),
        # prompts of a batch with pictures among their tokens, ragged, norms of each head's own
        dict(_append(16, 2000, 32, 8, 128, 128, 16, 900, 2000, "f16", "head", axes=3, prompt=True), name="append_pictures"),
        # two short questions behind the same instructions: the latency of a step
        dict(_shared(2, 1, 8, 8, 64, 16, 1000, 20, 30, 1, "f32", "beam"), name="shared_two"),
        # the headline batch after 40 steps, every source behind the same instructions
        dict(_shared(64, 20, 32, 8, 128, 16, 1500, 100, 700, 40, "bf16", "beam"), name="shared_beam"),
        # few questions about one long document
        dict(_shared(4, 8, 32, 8, 128, 64, 100000, 20, 300, 3, "f16", "beam"), name="shared_document"),
        # many answers searched for at once behind one long prompt, eight query heads to a head of the cache
        dict(_shared(128, 8, 32, 4, 128, 32, 8000, 10, 60, 12, "bf16", "beam"), name="shared_answers"),
        # the headline batch again: what its 20 branches looked at
        dict(_weigh(64, 20, 16, 16, 64, 16, 100, 700, 40, "bf16", "beam", True), name="weigh_beam"),
        # what the last 32 tokens of long prompts looked at, one score for all heads
        dict(_weigh(16, 32, 32, 8, 128, 32, 3000, 16000, 1, "f16", "chain", False), name="weigh_window"),
        # one sentence's cache cut to a quarter
        dict(_evict(1, 8, 64, 16, 1000, 1000, 0, 256, 4, 32, "f32", True), name="evict_one"),
        # the headline batch in the middle of a search: sources are cut, the tree of generated tokens stays
        dict(_evict(64, 8, 128, 16, 500, 1500, 800, 400, 4, 64, "bf16", True), name="evict_batch"),
        # long documents, one choice for all heads
        dict(_evict(4, 8, 128, 64, 50000, 65000, 24, 16384, 16, 512, "f16", False), name="evict_documents"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = 1.4e9
    while True:
        dtype = rng.choice(["f32", "f16", "bf16"])
        op = rng.choice(["append", "shared", "shared", "weigh", "evict"])
        B = _log(rng, 1, 128)
        D = rng.choice([32, 64, 80, 96, 128, 256])
        Hkv = rng.choice([1, 2, 4, 8])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
        page = rng.choice([8, 16, 32, 64, 128])
        lo = _log(rng, 1, 30000)
        hi = lo + _log(rng, 1, lo + 1)
        if op == "append":
            prompt = rng.random() < 0.4
            n = _log(rng, 1, 4000) if prompt else _log(rng, 1, 64)
            c = _append(B, n, Hq, Hkv, D, rng.choice([D, D, D // 32 * 16]), page, max(1, n // 2) if prompt else lo, n if prompt else hi, dtype,
                        rng.choice(["all", "all", "head", "none"]), 1, prompt, rng.random() < 0.3)
            c["axes"] = 3 if c["norm"] == "none" else rng.choice([1, 3])
        elif op == "evict":
            keep = _log(rng, 1, hi)
            c = _evict(B, Hkv, D, page, lo, hi, rng.choice([0, _log(rng, 1, 1000)]), keep, rng.randint(0, min(8, keep)),
                       rng.randint(0, keep // 2), dtype, rng.random() < 0.5)
        else:
            kind = rng.choice(["beam", "beam", "chain"])
            n = _log(rng, 1, 64) if kind == "beam" else _log(rng, 1, 300)
            steps = _log(rng, 1, 60) if kind == "beam" else 1
            if op == "shared":
                lo = _log(rng, 1, 3000)
                hi = lo + _log(rng, 1, lo + 1)
                common = _log(rng, 1, 100000)
                c = _shared(B, n, Hq, Hkv, D, page, common, lo, hi, steps, dtype, kind)
            else:
                common = 0
                c = _weigh(B, n, Hq, Hkv, D, page, lo, hi, steps, dtype, kind, rng.random() < 0.5)
            if (common + (lo + hi) / 2 + n * steps) * n * Hq * B > 2.8e8:      # the plain form holds every probability
                continue
        w = work(c)
        if w["bytes"] + w["flops"] / 100 <= largest and _pool_bytes(c) < 6e9:
            return c


def _lens(c):
    """Lengths from lo to hi, the same for every seed."""
    b = np.arange(c["B"], dtype=np.int64)
    return c["lo"] + (c["hi"] - c["lo"]) * ((b * 7919) % c["B"]) // max(1, c["B"] - 1)


def _pages_of(c):
    """(pages of a sentence, pages of what they have in common, pages of a sentence's new table)."""
    up = lambda x: -(-x // c["page"])
    if c["op"] == "append":
        return up(c["n"] if c["prompt"] else c["hi"] + c["n"]), 0, 0
    if c["op"] == "evict":
        return up(c["hi"] + c["tree"]), 0, up(min(c["keep"], c["hi"]) + c["tree"])
    return up(c["hi"] + c["n"] * c["steps"]), up(c["common"]) if c["op"] == "shared" else 0, 0


def _pool_bytes(c):
    per, common, new = _pages_of(c)
    return (c["B"] * (per + new) + common) * c["page"] * c["Hkv"] * c["D"] * ELEM[c["dtype"]] * 2


def work(case):
    e, B, Hkv, D = ELEM[case["dtype"]], case["B"], case["Hkv"], case["D"]
    lens = _lens(case)
    if case["op"] == "evict":
        H = Hkv if case["by_head"] else 1
        stay = int(np.minimum(lens, case["keep"]).sum()) + B * case["tree"]
        return {"bytes": stay * Hkv * D * e * 4 + int(lens.sum() + B * case["tree"]) * H * 8 + B * 8, "flops": 0}
    Hq, n = case["Hq"], case["n"]
    if case["op"] == "append":
        tokens = int(lens.sum()) if case["prompt"] else B * n
        return {"bytes": tokens * (Hq + 2 * Hkv) * D * e * 2 + tokens * 4 * (1 + case["axes"]),
                "flops": tokens * (Hq + Hkv) * (case["rot"] * 3 + (0 if case["norm"] == "none" else 4 * D))}
    tree = n * case["steps"]
    seen = case["steps"] if case["kind"] == "beam" else (n + 1) / 2
    held = int(lens.sum()) + B * tree
    asked = n * (float(lens.sum()) + B * seen)
    if case["op"] == "weigh":
        H = Hkv if case["by_head"] else 1
        return {"bytes": held * Hkv * D * e + held * H * 8 + B * n * Hq * (D * e + 4), "flops": int(2 * Hq * D * asked)}
    return {"bytes": (held + case["common"]) * Hkv * D * e * 2 + B * n * Hq * (D * e * 2 + 4),
            "flops": int(4 * Hq * D * (asked + n * B * case["common"]))}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _pages(case, dev, g):
    """A pool of pages and tables of them in random order."""
    B, page, Hkv, D, t = case["B"], case["page"], case["Hkv"], case["D"], TORCH[case["dtype"]]
    per, common, new = _pages_of(case)
    n_pages = B * (per + new) + common + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    k = torch.empty((n_pages, page, Hkv, D), dtype=t, device=dev).normal_(generator=g)
    v = torch.empty((n_pages, page, Hkv, D), dtype=t, device=dev).normal_(generator=g)
    return {"k_pages": k, "v_pages": v, "table": order[:B * per].reshape(B, per).contiguous(),
            "common": order[B * per:B * per + common].contiguous(), "new_table": order[B * per + common:n_pages - 3].reshape(B, new).contiguous()}


def _set_bit(words, slot):
    """words [B, n, W] int64, slot [n] int64: sets bit slot[i] in row i of every sentence."""
    W = words.shape[2]
    bit = torch.ones((), dtype=torch.int64, device=words.device) << (slot & 63)
    here = (torch.arange(W, device=words.device)[None, :] == (slot >> 6)[:, None])
    return words | torch.where(here, bit[:, None], 0)[None]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    B, Hkv, D, t = case["B"], case["Hkv"], case["D"], TORCH[case["dtype"]]
    lens = torch.from_numpy(_lens(case)).to(dev).to(torch.int32)
    st = _pages(case, dev, g) | {"case": case}
    if case["op"] == "append":
        n, Hq, axes = case["n"], case["Hq"], case["axes"]
        for name, h in (("q", Hq), ("k", Hkv), ("v", Hkv)):            # heads of different sizes, as products of weights leave them
            size = torch.rand((h, 1), generator=g, device=dev) * 4 + 0.1
            st[name] = torch.empty((B, n, h, D), dtype=t, device=dev).normal_(generator=g).mul_(size.to(t))
            if name != "v":
                w = torch.rand((D,) if case["norm"] == "all" else (h, D), generator=g, device=dev) + 0.5
                st[name + "_weight"] = None if case["norm"] == "none" else w.to(t)
        st["q_out"] = torch.zeros((B, n, Hq, D), dtype=t, device=dev)
        st["inv_freq"] = (10000.0 ** (-torch.arange(0, case["rot"], 2, device=dev, dtype=torch.float64) / case["rot"])).float()
        st |= {"first": torch.zeros_like(lens), "count": lens} if case["prompt"] else {"first": lens, "count": None}
        i = torch.arange(n, device=dev, dtype=torch.int32)[None, :].expand(B, n)
        if axes == 3:                                       # a text of 100 tokens, then frames of 20 x 30 places
            at = (i - 100).clamp(min=0)
            time = st["first"][:, None] + torch.where(i < 100, i, 100 + at // 600)
            st["position"] = torch.stack((time, torch.where(i < 100, time, 100 + at % 600 // 30), torch.where(i < 100, time, 100 + at % 30)), dim=2).contiguous()
            st["axis"] = torch.arange(case["rot"] // 2, device=dev, dtype=torch.int32) % 3
        else:
            depth = torch.randint(1, 100, (B, 1), generator=g, device=dev, dtype=torch.int32)
            st["position"] = None if case["prompt"] else (lens[:, None] + depth).expand(B, n).contiguous()
            st["axis"] = None
        return st
    if case["op"] == "evict":
        H, width = Hkv if case["by_head"] else 1, case["hi"] + case["tree"]
        score = torch.empty((B, H, width), device=dev).exponential_(generator=g).pow_(3)
        st["score"] = score.masked_fill_(torch.rand((B, H, width), generator=g, device=dev) < 0.05, 0.0)       # what nobody looked at
        return st | {"prefix": lens, "tree": torch.full_like(lens, case["tree"]), "max_len": width}
    n, Hq, steps = case["n"], case["Hq"], case["steps"]
    tree = n * steps
    st["q"] = torch.empty((B, n, Hq, D), dtype=t, device=dev).normal_(generator=g)
    st |= {"prefix": lens, "tree": torch.full_like(lens, tree), "mask": None, "max_len": case["hi"] + tree}
    if case["kind"] == "beam":
        rows = torch.arange(n, device=dev)
        words = torch.zeros((B, n, -(-tree // 64)), dtype=torch.int64, device=dev)
        for s in range(steps):
            back = torch.randint(0, n, (B, n, 1), generator=g, device=dev).expand(-1, -1, words.shape[2])
            words = _set_bit(words.gather(1, back) if s else words, s * n + rows)
        st["mask"] = words
    if case["op"] == "shared":
        return st | {"common_len": torch.full((1,), case["common"], dtype=torch.int32, device=dev)}
    st["score"] = torch.rand((B, Hkv if case["by_head"] else 1, st["max_len"]), generator=g, device=dev)
    st["lse"] = torch.empty((B, n, Hq), device=dev)         # the attention before has left it
    seen = _seen(st)
    for b in range(B):
        k = st["k_pages"][st["table"][b].long()].flatten(0, 1)[:st["max_len"]].float().permute(1, 2, 0).contiguous()       # [Hkv, D, L]
        s = torch.matmul(st["q"][b].float().reshape(n, Hkv, Hq // Hkv, D).permute(1, 0, 2, 3).reshape(Hkv, -1, D), k) * D ** -0.5
        s = s.reshape(Hkv, n, Hq // Hkv, -1).masked_fill(~seen[b][None, :, None], -math.inf)
        st["lse"][b] = torch.logsumexp(s, dim=3).permute(1, 0, 2).reshape(n, Hq)
    return st


# ---- the operators ---------------------------------------------------------------------------------------------------

def _seen(st):
    """[B, n, L]: which of its sentence's tokens a node sees."""
    n, dev = st["case"]["n"], st["prefix"].device
    j = torch.arange(st["max_len"], device=dev)[None, None, :] - st["prefix"][:, None, None]
    if st["mask"] is None:
        seen = j <= st["tree"][:, None, None] - n + torch.arange(n, device=dev)[None, :, None]
    else:
        bit = j.clamp(0, 64 * st["mask"].shape[2] - 1).expand(-1, n, -1)
        seen = ((st["mask"].gather(2, bit >> 6) >> (bit & 63)) & 1).bool() | (j < 0)
    return seen & (j < st["tree"][:, None, None])


def _by_head(x, Hkv):
    """[B, n, Hq, D] as [B, Hkv, n * G, D] in 32 bits."""
    B, n, Hq, D = x.shape
    return x.float().reshape(B, n, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * (Hq // Hkv), D)


def _turned(st, x, weight):
    c = st["case"]
    y = x.float()
    if weight is not None:
        y = y * (y.square().mean(dim=-1, keepdim=True) + EPS).rsqrt() * weight.float()
    position = st["position"]
    if position is None:
        position = st["first"][:, None] + torch.arange(c["n"], device=x.device)[None, :]
    position = position[:, :, None] if st["axis"] is None else position[:, :, st["axis"].long()]
    angle = position.double() * st["inv_freq"].double()     # 64 bits: far positions
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    rot = c["rot"]
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if c["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    p, q = a * cos - b * sin, b * cos + a * sin
    z = torch.stack((p, q), dim=-1).flatten(-2) if c["interleaved"] else torch.cat((p, q), dim=-1)
    return torch.cat((z, y[..., rot:]), dim=-1).to(x.dtype)


def _plain_append(st):
    c = st["case"]
    n, page = c["n"], c["page"]
    i = torch.arange(n, device=st["k"].device)[None, :]
    rows = torch.arange(c["B"], device=i.device)[:, None]
    src = i if st["count"] is None else torch.where(i < st["count"][:, None], i, 0)  # absent tokens write the first once more
    at = (st["first"][:, None] + src).long()
    slot = st["table"].gather(1, at // page).long() * page + at % page
    st["k_pages"].view(-1, c["Hkv"], c["D"])[slot.flatten()] = _turned(st, st["k"], st["k_weight"])[rows, src].flatten(0, 1)
    st["v_pages"].view(-1, c["Hkv"], c["D"])[slot.flatten()] = st["v"][rows, src].flatten(0, 1)
    q = _turned(st, st["q"], st["q_weight"])
    if st["count"] is not None:
        q = torch.where((i < st["count"][:, None])[:, :, None, None], q, 0)
    st["q_out"].copy_(q)
    return st["q_out"], st["k_pages"], st["v_pages"]


def _plain_shared(st):
    c = st["case"]
    B, n, Hq, Hkv, D, P, L = c["B"], c["n"], c["Hq"], c["Hkv"], c["D"], c["common"], st["max_len"]
    G, table, common = Hq // Hkv, st["table"].long(), st["common"].long()
    q = _by_head(st["q"], Hkv) * D ** -0.5
    k = st["k_pages"][common].flatten(0, 1)[:P].float().permute(1, 2, 0).contiguous()                   # [Hkv, D, P]
    v = st["v_pages"][common].flatten(0, 1)[:P].float().permute(1, 0, 2).contiguous()
    s = torch.matmul(q.transpose(0, 1).reshape(Hkv, B * n * G, D), k)
    own_k = st["k_pages"][table].flatten(1, 2)[:, :L].float().permute(0, 2, 3, 1).contiguous()          # [B, Hkv, D, L]
    own_v = st["v_pages"][table].flatten(1, 2)[:, :L].float().permute(0, 2, 1, 3).contiguous()
    r = torch.matmul(q, own_k).reshape(B, Hkv, n, G, L).masked_fill_(~_seen(st)[:, None, :, None, :], -math.inf).reshape(B, Hkv, n * G, L)
    top = torch.maximum(s.amax(dim=2).reshape(Hkv, B, n * G).transpose(0, 1), r.amax(dim=3))            # [B, Hkv, n * G]
    s = s.sub_(top.transpose(0, 1).reshape(Hkv, -1, 1)).exp_()
    r = r.sub_(top[..., None]).exp_()
    total = s.sum(dim=2).reshape(Hkv, B, n * G).transpose(0, 1) + r.sum(dim=3)
    o = torch.matmul(s, v).reshape(Hkv, B, n * G, D).transpose(0, 1) + torch.matmul(r, own_v)
    o = (o / total[..., None]).reshape(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    return o.to(st["q"].dtype), (top + total.log()).reshape(B, Hkv, n, G).permute(0, 2, 1, 3).reshape(B, n, Hq)


def _plain_weigh(st):
    c = st["case"]
    B, n, Hq, Hkv, D, L = c["B"], c["n"], c["Hq"], c["Hkv"], c["D"], st["max_len"]
    k = st["k_pages"][st["table"].long()].flatten(1, 2)[:, :L].float().permute(0, 2, 3, 1).contiguous()
    s = torch.matmul(_by_head(st["q"], Hkv), k).mul_(D ** -0.5).reshape(B, Hkv, n, Hq // Hkv, L)
    lse = st["lse"].reshape(B, n, Hkv, Hq // Hkv).permute(0, 2, 1, 3)[..., None]
    w = s.sub_(lse).exp_().masked_fill_(~_seen(st)[:, None, :, None, :], 0.0).sum(dim=(2, 3))
    return st["score"] + (w if c["by_head"] else w.sum(dim=1, keepdim=True))


def _plain_evict(st):
    c = st["case"]
    B, page, Hkv, D, tree, L = c["B"], c["page"], c["Hkv"], c["D"], c["tree"], st["max_len"]
    score, H = st["score"], st["score"].shape[1]
    dev = score.device
    t = torch.arange(L, device=dev)[None, None, :]
    prefix = st["prefix"].long()[:, None, None]
    rank = score.view(torch.int32).long() + 1               # scores are not negative: their bits are in their order
    rank = torch.where((t < c["sinks"]) | (t >= prefix - c["recent"]), rank + (1 << 32), rank)
    rank = torch.where(t < prefix, rank, 0)
    order = rank.sort(dim=2, descending=True, stable=True).indices
    stay = prefix.clamp(max=c["keep"])
    chosen = torch.zeros((B, H, L), dtype=torch.bool, device=dev).scatter_(2, order, (t < stay).expand(B, H, L))
    chosen |= (t >= prefix) & (t < prefix + tree)
    src = torch.where(chosen, t, L).sort(dim=2).values[:, :, :min(c["keep"], c["hi"]) + tree]          # old places, first to last, then L
    there, src = src < L, src.clamp(max=L - 1)
    moved = torch.zeros_like(score)
    moved[:, :, :src.shape[2]] = torch.where(there, score.gather(2, src), 0.0)
    j = torch.arange(src.shape[2], device=dev)
    new = (st["new_table"].long()[:, j // page] * page + j % page)[:, None, :].expand(B, Hkv, -1)
    src, there = src.expand(B, Hkv, -1), there.expand(B, Hkv, -1)
    old = st["table"].long().gather(1, (src // page).flatten(1)).reshape(src.shape) * page + src % page
    head = torch.arange(Hkv, device=dev)[None, :, None].expand(B, Hkv, src.shape[2])
    old, new, head = old[there], new[there], head[there]
    for pages in (st["k_pages"].view(-1, Hkv, D), st["v_pages"].view(-1, Hkv, D)):
        pages[new, head] = pages[old, head]
    return st["k_pages"], st["v_pages"], stay[:, 0, 0].int(), moved


def run(state):
    st, op = state, state["case"]["op"]
    if not own:
        return {"append": _plain_append, "shared": _plain_shared, "weigh": _plain_weigh, "evict": _plain_evict}[op](st)
    from paper_1804_06609_amd import beam
    c, k_pages, v_pages, table = st["case"], st["k_pages"], st["v_pages"], st["table"]
    if op == "append":
        q = beam.append(st["k"], st["v"], k_pages, v_pages, table, st["first"], st["count"], position=st["position"], axis=st["axis"],
                        inv_freq=st["inv_freq"], interleaved=c["interleaved"], q=st["q"], q_out=st["q_out"],
                        eps=None if c["norm"] == "none" else EPS, q_weight=st["q_weight"], k_weight=st["k_weight"])
        return q, k_pages, v_pages
    if op == "shared":
        return beam.attend_shared(st["q"], k_pages, v_pages, st["common"], st["common_len"], table, st["prefix"], st["tree"], st["mask"],
                                  max_shared=c["common"], max_len=st["max_len"], return_lse=True)
    if op == "weigh":
        return beam.weigh(st["score"], st["q"], st["lse"], k_pages, table, st["prefix"], st["tree"], st["mask"], max_len=st["max_len"],
                          out=torch.empty_like(st["score"]))
    stay, moved = beam.evict(st["score"], k_pages, v_pages, table, st["new_table"], st["prefix"], st["tree"], keep=c["keep"], sinks=c["sinks"],
                             recent=c["recent"], max_len=st["max_len"])
    return k_pages, v_pages, stay, moved


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _exact_append(st):
    c = st["case"]
    rot, page = c["rot"], c["page"]
    dev = st["q"].device
    q_out = torch.zeros(st["q"].shape, dtype=torch.float64, device=dev)
    k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
    first, table = st["first"].tolist(), st["table"].tolist()
    pairs = torch.arange(rot // 2, device=dev)
    lo, hi = (2 * pairs, 2 * pairs + 1) if c["interleaved"] else (pairs, pairs + rot // 2)
    for b in range(c["B"]):
        n = c["n"] if st["count"] is None else st["count"].tolist()[b]
        if st["position"] is None:
            pos = torch.arange(first[b], first[b] + n, device=dev)[:, None].expand(n, rot // 2)
        elif st["axis"] is None:
            pos = st["position"][b, :n, None].expand(n, rot // 2)
        else:
            pos = torch.stack([st["position"][b, :n, a] for a in st["axis"].tolist()], dim=1)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=dev), pos.double() * st["inv_freq"].double())[:, None]

        def normed(x, weight):
            y = x[:n].double()
            if weight is not None:
                y = y / (torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 / c["D"] + EPS).sqrt() * weight.double()
            z = torch.complex(y[..., lo], y[..., hi]) * turn
            y[..., lo], y[..., hi] = z.real, z.imag
            return y

        q_out[b, :n] = normed(st["q"][b], st["q_weight"])
        at = np.arange(first[b], first[b] + n)
        page_of = torch.tensor([table[b][p] for p in at // page], device=dev)
        k_pages[page_of, torch.from_numpy(at % page).to(dev)] = normed(st["k"][b], st["k_weight"])
        v_pages[page_of, torch.from_numpy(at % page).to(dev)] = st["v"][b, :n].double()
    return q_out, k_pages, v_pages


def _hidden(st, b):
    """[n, tokens] of sentence b: what its nodes do not see."""
    n, prefix, tree = st["case"]["n"], int(st["prefix"][b]), int(st["tree"][b])
    seen = np.ones((n, prefix + tree), bool)
    if st["mask"] is None:
        seen[:, prefix:] = np.tri(n, tree, tree - n, dtype=bool)
    else:
        bits = np.unpackbits(st["mask"][b].cpu().numpy().view(np.uint8), axis=1, bitorder="little")
        seen[:, prefix:] = bits[:, :tree].astype(bool)
    return torch.from_numpy(~seen).to(st["q"].device)


def _exact_shared(st):
    c = st["case"]
    G, D, P = c["Hq"] // c["Hkv"], c["D"], c["common"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    lse = torch.zeros(st["q"].shape[:3], dtype=torch.float64, device=out.device)
    for h in range(c["Hkv"]):
        common = [st[x][st["common"].long(), :, h].reshape(-1, D)[:P].double() for x in ("k_pages", "v_pages")]
        for b in range(c["B"]):
            hidden = _hidden(st, b)
            L = hidden.shape[1]
            pages = st["table"][b, :-(-L // c["page"])].long()
            k, v = (torch.cat((x, st[name][pages, :, h].reshape(-1, D)[:L].double())) for x, name in zip(common, ("k_pages", "v_pages")))
            s = st["q"][b, :, h * G:h * G + G].double().transpose(0, 1) @ k.t() / math.sqrt(D)         # [G, n, P + L]
            s[:, :, P:].masked_fill_(hidden[None], -math.inf)
            w = s.softmax(dim=2)
            lse[b, :, h * G:h * G + G] = torch.logsumexp(s, dim=2).t()
            out[b, :, h * G:h * G + G] = (w @ v).transpose(0, 1)
    return out, lse


def _exact_weigh(st):
    c = st["case"]
    G = c["Hq"] // c["Hkv"]
    score = st["score"].double()
    for b in range(c["B"]):
        hidden = _hidden(st, b)
        L = hidden.shape[1]
        pages = st["table"][b, :-(-L // c["page"])].long()
        for h in range(c["Hq"]):
            k = st["k_pages"][pages, :, h // G].reshape(-1, c["D"])[:L].double()
            x = st["q"][b, :, h].double() @ k.t() / math.sqrt(c["D"]) - st["lse"][b, :, h, None].double()
            score[b, h // G if c["by_head"] else 0, :L] += torch.where(hidden, 0.0, x.exp()).sum(dim=0)
    return score


def _exact_evict(st):
    c = st["case"]
    H, page, tree = st["score"].shape[1], c["page"], c["tree"]
    k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
    score, table, new_table = st["score"].cpu().numpy(), st["table"].cpu().numpy(), st["new_table"].cpu().numpy()
    prefix = st["prefix"].tolist()
    moved, stay = np.zeros(score.shape), [min(c["keep"], p) for p in prefix]
    for b in range(c["B"]):
        t = np.arange(prefix[b])
        last = (t >= c["sinks"]) & (t < prefix[b] - c["recent"])
        for h in range(H):
            kept = np.sort(np.lexsort((t, -score[b, h, :prefix[b]], last))[:stay[b]])
            kept = np.concatenate((kept, np.arange(prefix[b], prefix[b] + tree)))
            j = np.arange(len(kept))
            moved[b, h, j] = score[b, h, kept]
            of = slice(None) if H == 1 else slice(h, h + 1)
            to, at = (torch.from_numpy(x).to(k_pages.device) for x in (new_table[b, j // page].astype(np.int64), j % page))
            frm, was = (torch.from_numpy(x).to(k_pages.device) for x in (table[b, kept // page].astype(np.int64), kept % page))
            for pages in (k_pages, v_pages):
                pages[to, at, of] = pages[frm, was, of]
    return k_pages, v_pages, stay, moved


def exact(case, seed):
    st = prepare(case, seed)
    out = {"append": _exact_append, "shared": _exact_shared, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](st)
    if case["op"] == "evict":
        dev = out[0].device
        return out[0], out[1], torch.tensor(out[2], dtype=torch.int32, device=dev), torch.from_numpy(out[3]).to(dev)
    return out
