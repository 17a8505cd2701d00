"""Workloads by which the speed of the operators around a beam-search step is measured.

A decoder that searches with a beam does four things next to its layers' products, once per time step: it rotates the
new keys and puts them into a paged cache (`append`), attends over that cache, where the hypotheses of a sentence are
the branches of a tree of cached tokens (`attend`), chooses the new beam from the logits (`select`), and lets its
states follow the back-pointers (`reorder`).  The inputs stand in for a decoder's: logits are N(0,1) with a Zipf
bias, ancestor masks come from a search that was played through, pages lie in the pool in random order.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

ELEM = {"f32": 4, "f16": 2, "bf16": 2}
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
PAD, EOS = 0, 2
FINISHED, DEAD = 1, 2


def _select(B, k, k_out, V, dtype):
    return {"op": "select", "B": B, "k": k, "k_out": k_out, "V": V, "dtype": dtype}


def _reorder(B, k, states, heads, cap, live, width, dtype):
    """`states` tensors [B, k, heads, cap, width] of which the first `live` places of the fourth axis are in use."""
    return {"op": "reorder", "B": B, "k": k, "states": states, "heads": heads, "cap": cap, "live": live, "width": width, "dtype": dtype}


def _append(B, n, Hq, Hkv, D, rot, page, lo, hi, dtype, prompt=False, interleaved=False):
    """n tokens a sentence behind lo..hi cached ones; prompt: ragged counts from the cache's start, chain positions."""
    return {"op": "append", "B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot, "page": page, "lo": lo, "hi": hi,
            "dtype": dtype, "prompt": prompt, "interleaved": interleaved}


def _attend(B, n, Hq, Hkv, D, page, lo, hi, steps, dtype, kind):
    """lo..hi shared tokens a sentence.  kind "beam": behind them `steps` tokens for each of n beam slots, a query per slot;
    "draft": n drafted tokens, each behind a random earlier one, all asking; "chain": n tokens in a row, all asking."""
    return {"op": "attend", "B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "lo": lo, "hi": hi, "steps": steps,
            "dtype": dtype, "kind": kind}


def listed():
    return [
        # one sentence, a toy vocabulary, beam 5: launches and latencies only
        dict(_select(1, 5, 5, 1000, "f32"), name="select_toy"),
        # a vocabulary whose rows start on no 16 bytes
        dict(_select(24, 7, 7, 50001, "f16"), name="select_odd_vocab"),
        # the library's headline shape, and its widest beam from a decoder that hands over bf16
        dict(_select(64, 20, 20, 32000, "f32"), name="select_batch64"),
        dict(_select(128, 64, 64, 50000, "bf16"), name="select_wide_beam"),
        # the recurrent state of one sentence's beam (output and memory of two layers)
        dict(_reorder(1, 5, 4, 1, 1, 1, 512, "f32"), name="reorder_recurrent"),
        # dense caches of a six-layer decoder, keys and values, in the middle of a decode
        dict(_reorder(64, 20, 12, 8, 100, 57, 64, "bf16"), name="reorder_dense_caches"),
        # a time step of the headline batch: 20 new tokens a sentence behind a source and what has been generated
        dict(_append(64, 20, 32, 8, 128, 128, 16, 300, 1500, "bf16"), name="append_beam"),
        # prompts of a batch, ragged, half of each head rotated
        dict(_append(16, 2000, 32, 8, 128, 64, 64, 900, 2000, "f16", prompt=True), name="append_prompts"),
        # one sentence, one hypothesis: the latency of a decoding step
        dict(_attend(1, 1, 8, 8, 64, 16, 1000, 1000, 1, "f32", "beam"), name="attend_one_token"),
        # the headline batch after 40 steps: 20 branches a sentence over a shared source
        dict(_attend(64, 20, 16, 16, 64, 16, 100, 700, 40, "bf16", "beam"), name="attend_beam"),
        # few sentences over long documents
        dict(_attend(4, 8, 32, 8, 128, 64, 50000, 65000, 3, "bf16", "beam"), name="attend_long"),
        # drafts of 63 tokens verified at once, eight query heads to a head of the cache
        dict(_attend(32, 63, 32, 4, 128, 16, 500, 4000, 1, "f16", "draft"), name="attend_draft"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = 1.4e9
    while True:
        dtype = rng.choice(["f32", "f16", "bf16"])
        op = rng.choice(["select", "reorder", "append", "attend", "attend"])
        B = _log(rng, 1, 128)
        if op == "select":
            k = _log(rng, 1, 64)
            k_out = rng.choice([k, k, min(64, 2 * k), _log(rng, 1, 64)])
            c = _select(B, k, k_out, _log(rng, 200, 130000), dtype)
            if c["V"] < 2 * k_out or B * k * c["V"] > 4.0e8:
                continue
        elif op == "reorder":
            cap = _log(rng, 1, 300)
            c = _reorder(B, _log(rng, 1, 64), rng.randint(1, 16), rng.choice([1, 4, 8, 12]), cap, rng.randint(1, cap),
                         rng.choice([40, 64, 80, 128, 513]), dtype)
        else:
            D = rng.choice([32, 64, 80, 96, 128, 256])
            Hkv = rng.choice([1, 2, 4, 8])
            Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
            page = rng.choice([8, 16, 32, 64, 128])
            lo = _log(rng, 1, 30000)
            hi = lo + _log(rng, 1, lo + 1)
            if op == "append":
                prompt = rng.random() < 0.4
                n = _log(rng, 1, 4000) if prompt else _log(rng, 1, 64)
                c = _append(B, n, Hq, Hkv, D, rng.choice([D, D, D // 16 * 8 if D % 32 else D // 2]), page,
                            max(1, n // 2) if prompt else lo, n if prompt else hi, dtype, prompt, rng.random() < 0.3)
                if c["rot"] % 16:
                    continue
            else:
                kind = rng.choice(["beam", "beam", "draft", "chain"])
                n = _log(rng, 1, 64) if kind != "chain" else _log(rng, 1, 1500)
                c = _attend(B, n, Hq, Hkv, D, page, lo, hi, _log(rng, 1, 60) if kind == "beam" else 1, dtype, kind)
                if (lo + hi) / 2 * n * Hq * B > 2.5e8:      # the plain form holds every probability
                    continue
        w = work(c)
        if w["bytes"] + w["flops"] / 100 <= largest:
            return c


def _lens(c):
    """Lengths from lo to hi, the same for every seed."""
    b = np.arange(c["B"], dtype=np.int64)
    return c["lo"] + (c["hi"] - c["lo"]) * ((b * 7919) % c["B"]) // max(1, c["B"] - 1)


def work(case):
    e, B = ELEM[case["dtype"]], case["B"]
    if case["op"] == "select":
        k, V = case["k"], case["V"]
        return {"bytes": B * k * (V * e + 5) + B * case["k_out"] * 13, "flops": 4 * B * k * V}
    if case["op"] == "reorder":
        row = case["states"] * case["heads"] * case["live"] * case["width"] * e
        k = case["k"]
        distinct = k * (1 - (1 - 1 / k) ** k)               # of k random parents
        return {"bytes": int(B * (k + distinct) * row) + B * k * 4, "flops": 0}
    Hq, Hkv, D, n = case["Hq"], case["Hkv"], case["D"], case["n"]
    if case["op"] == "append":
        tokens = int(_lens(case).sum()) if case["prompt"] else B * n
        return {"bytes": tokens * (Hq + 2 * Hkv) * D * e * 2 + tokens * 8, "flops": tokens * (Hq + Hkv) * case["rot"] * 3}
    P = int(_lens(case).sum())
    tree = n * case["steps"]
    seen = case["steps"] if case["kind"] == "beam" else (n + 1) / 2 if case["kind"] == "chain" else 1 + math.log(n)
    return {"bytes": (P + B * tree) * Hkv * D * e * 2 + B * n * Hq * (D * e * 2 + 4),
            "flops": int(4 * Hq * D * n * (P + B * seen))}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _pages(case, dev, g, capacity):
    """A pool of pages and a table of them in random order."""
    B, page, Hkv, D, t = case["B"], case["page"], case["Hkv"], case["D"], TORCH[case["dtype"]]
    per = -(-capacity // page)
    n_pages = B * per + 3
    table = torch.randperm(n_pages, generator=g, device=dev)[:B * per].to(torch.int32).reshape(B, per).contiguous()
    k = torch.empty((n_pages, page, Hkv, D), dtype=t, device=dev).normal_(generator=g)
    v = torch.empty((n_pages, page, Hkv, D), dtype=t, device=dev).normal_(generator=g)
    return {"k_pages": k, "v_pages": v, "table": table}


def _set_bit(words, slot):
    """words [B, n, W] int64, slot [n] int64: sets bit slot[i] in row i of every sentence."""
    W = words.shape[2]
    bit = torch.ones((), dtype=torch.int64, device=words.device) << (slot & 63)
    here = (torch.arange(W, device=words.device)[None, :] == (slot >> 6)[:, None])
    return words | torch.where(here, bit[:, None], 0)[None]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    B, t = case["B"], TORCH[case["dtype"]]
    if case["op"] == "select":
        k, V = case["k"], case["V"]
        bias = 1.0 / torch.arange(1, V + 1, device=dev, dtype=torch.float32).pow(1.1) * 8.0
        logits = torch.empty((B, k, V), dtype=t, device=dev)
        for b in range(B):
            x = torch.empty((k, V), device=dev).normal_(generator=g)
            logits[b] = (x + bias[torch.randperm(V, generator=g, device=dev)]).to(t)
        score = -torch.rand((B, k), generator=g, device=dev).mul_(4.0).add_(6.0).sort(dim=1).values
        flags = (torch.rand((B, k), generator=g, device=dev) < 0.1).to(torch.uint8) * FINISHED
        dead = (torch.arange(k, device=dev)[None, :] >= k - k // 8) & (torch.arange(B, device=dev)[:, None] % 3 == 1)
        flags = torch.where(dead, torch.full_like(flags, DEAD), flags)
        score = torch.where(dead, torch.full_like(score, -math.inf), score)
        return {"case": case, "logits": logits, "score": score, "flags": flags}
    if case["op"] == "reorder":
        k = case["k"]
        shape = (B, k, case["heads"], case["cap"], case["width"])
        src = [torch.empty(shape, dtype=t, device=dev).normal_(generator=g) for _ in range(case["states"])]
        dst = [torch.zeros(shape, dtype=t, device=dev) for _ in range(case["states"])]
        back = torch.randint(0, k, (B, k), generator=g, device=dev, dtype=torch.int32)
        back[:, k - k // 10:] = torch.where(torch.arange(B, device=dev)[:, None] % 4 == 1, -1, back[:, k - k // 10:])  # empty slots
        live = case["live"]
        return {"case": case, "back": back, "src": [x[:, :, :, :live] for x in src], "dst": [x[:, :, :, :live] for x in dst]}
    lens = torch.from_numpy(_lens(case)).to(dev).to(torch.int32)
    n, Hq, Hkv, D = case["n"], case["Hq"], case["Hkv"], case["D"]
    if case["op"] == "append":
        st = _pages(case, dev, g, case["n"] if case["prompt"] else case["hi"] + n)
        st |= {name: torch.empty((B, n, h, D), dtype=t, device=dev).normal_(generator=g) for name, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
        st["q_out"] = torch.zeros((B, n, Hq, D), dtype=t, device=dev)
        st["inv_freq"] = (10000.0 ** (-torch.arange(0, case["rot"], 2, device=dev, dtype=torch.float64) / case["rot"])).float()
        if case["prompt"]:
            st |= {"first": torch.zeros_like(lens), "count": lens, "position": None}
        else:                                               # a beam's tokens all have the same depth; the slots go on
            depth = torch.randint(1, 100, (B, 1), generator=g, device=dev, dtype=torch.int32)
            st |= {"first": lens, "count": None, "position": (lens[:, None] + depth).expand(B, n).contiguous()}
        return st | {"case": case}
    steps, kind = case["steps"], case["kind"]
    tree = n * steps
    st = _pages(case, dev, g, case["hi"] + tree)
    st["q"] = torch.empty((B, n, Hq, D), dtype=t, device=dev).normal_(generator=g)
    st |= {"case": case, "prefix": lens, "tree": torch.full_like(lens, tree), "mask": None, "max_len": case["hi"] + tree}
    rows = torch.arange(n, device=dev)
    if kind == "beam":
        words = torch.zeros((B, n, -(-tree // 64)), dtype=torch.int64, device=dev)
        for s in range(steps):
            back = torch.randint(0, n, (B, n, 1), generator=g, device=dev).expand(-1, -1, words.shape[2])
            words = _set_bit(words.gather(1, back) if s else words, s * n + rows)
        st["mask"] = words
    elif kind == "draft":
        words = _set_bit(torch.zeros((B, n, -(-n // 64)), dtype=torch.int64, device=dev), rows)
        for i in range(1, n):
            parent = torch.randint(0, i, (B, 1, 1), generator=g, device=dev).expand(-1, -1, words.shape[2])
            words[:, i] |= words.gather(1, parent)[:, 0]
        st["mask"] = words
    return st


# ---- the operators ---------------------------------------------------------------------------------------------------

def _plain_select(st):
    c = st["case"]
    B, k, V, m = c["B"], c["k"], c["V"], c["k_out"]
    x = st["logits"].double()                               # 64 bits: beams are compared across rows, next to each other
    top = x.amax(dim=2, keepdim=True)
    s = x - (top + (x - top).exp().sum(dim=2, keepdim=True).log()) + st["score"].double()[:, :, None]
    ids = torch.arange(V, device=x.device)
    over = (st["flags"] & FINISHED).bool()[:, :, None]
    s = torch.where(over, torch.where(ids == PAD, st["score"].double()[:, :, None], -math.inf), s)
    s = torch.where((st["flags"] & DEAD).bool()[:, :, None], -math.inf, s).reshape(B, k * V)
    least = s.topk(m, dim=1).values[:, -1:]                 # the last score that is in; of its equals the first ones
    more, same = s > least, s == least
    chosen = more | (same & (same.cumsum(dim=1) <= m - more.sum(dim=1, keepdim=True)))
    flat = torch.where(chosen, k * V - torch.arange(k * V, device=x.device), -1).topk(m, dim=1).values
    flat = k * V - flat                                     # ascending
    s, order = s.gather(1, flat).sort(dim=1, descending=True, stable=True)
    flat = flat.gather(1, order)
    found = s > -math.inf
    back = flat // V
    token = torch.where(found, flat - back * V, PAD).int()
    flags = torch.where((token == EOS) | (st["flags"].gather(1, back) & FINISHED).bool(), FINISHED, 0)
    return (token, torch.where(found, back, -1).int(), torch.where(found, s, -math.inf).float(),
            torch.where(found, flags, DEAD).to(torch.uint8))


def _plain_reorder(st):
    back = st["back"].long()
    rows = torch.arange(back.shape[0], device=back.device)[:, None]
    there = (back >= 0)[:, :, None, None, None]
    return [d.copy_(torch.where(there, s[rows, back.clamp(min=0)], 0)) for s, d in zip(st["src"], st["dst"])]


def _rotated(x, position, inv_freq, interleaved):
    angle = position.double()[:, :, None] * inv_freq.double()           # 64 bits: far positions
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    rot = 2 * inv_freq.numel()
    y = x[..., :rot].float()
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:])
    p, q = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((p, q), dim=-1).flatten(-2) if interleaved else torch.cat((p, q), dim=-1)
    return torch.cat((y.to(x.dtype), x[..., rot:]), dim=-1)


def _plain_append(st):
    c = st["case"]
    n, page = c["n"], c["page"]
    i = torch.arange(n, device=st["k"].device)[None, :]
    rows = torch.arange(c["B"], device=i.device)[:, None]
    src = i if st["count"] is None else torch.where(i < st["count"][:, None], i, 0)  # absent tokens write the first once more
    position = st["first"][:, None] + i if st["position"] is None else st["position"]
    at = (st["first"][:, None] + src).long()
    slot = st["table"].gather(1, at // page).long() * page + at % page
    k = _rotated(st["k"], position, st["inv_freq"], c["interleaved"])
    st["k_pages"].view(-1, c["Hkv"], c["D"])[slot.flatten()] = k[rows, src].flatten(0, 1)
    st["v_pages"].view(-1, c["Hkv"], c["D"])[slot.flatten()] = st["v"][rows, src].flatten(0, 1)
    q = _rotated(st["q"], position, st["inv_freq"], c["interleaved"])
    if st["count"] is not None:
        q = torch.where((i < st["count"][:, None])[:, :, None, None], q, 0)
    st["q_out"].copy_(q)
    return st["q_out"], st["k_pages"], st["v_pages"]


def _plain_attend(st):
    c = st["case"]
    B, n, Hq, Hkv, D, L = c["B"], c["n"], c["Hq"], c["Hkv"], c["D"], st["max_len"]
    G, dev = Hq // Hkv, st["q"].device
    table = st["table"].long()
    k = st["k_pages"][table].flatten(1, 2)[:, :L].float().permute(0, 2, 3, 1).contiguous()      # [B, Hkv, D, L]
    v = st["v_pages"][table].flatten(1, 2)[:, :L].float().permute(0, 2, 1, 3).contiguous()
    q = st["q"].float().reshape(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    s = torch.matmul(q, k).reshape(B, Hkv, n, G, L) * D ** -0.5
    j = torch.arange(L, device=dev)[None, None, :] - st["prefix"][:, None, None]                # [B, 1, L]
    i = torch.arange(n, device=dev)[None, :, None]
    if st["mask"] is None:
        seen = j <= st["tree"][:, None, None] - n + i
    else:
        bit = j.clamp(0, 64 * st["mask"].shape[2] - 1).expand(B, n, L)
        seen = ((st["mask"].gather(2, bit >> 6) >> (bit & 63)) & 1).bool() | (j < 0)
    seen = seen & (j < st["tree"][:, None, None])
    s = s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = s.amax(dim=4, keepdim=True).clamp(min=-3.0e38)
    p = s.sub_(top).exp_()
    total = p.sum(dim=4, keepdim=True)
    o = torch.matmul(p.reshape(B, Hkv, n * G, L), v).reshape(B, Hkv, n, G, D) / total.clamp(min=1e-37)
    out = o.permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D).to(st["q"].dtype)
    return out, (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, n, Hq)


def run(state):
    st, op = state, state["case"]["op"]
    if not own:
        return {"select": _plain_select, "reorder": _plain_reorder, "append": _plain_append, "attend": _plain_attend}[op](st)
    from paper_1804_06609_amd import beam
    if op == "select":
        return beam.select(st["logits"], st["score"], st["flags"], st["case"]["k_out"], EOS, PAD)
    if op == "reorder":
        return beam.reorder(st["back"], st["src"], st["dst"])
    if op == "append":
        q = beam.append(st["k"], st["v"], st["k_pages"], st["v_pages"], st["table"], st["first"], st["count"], position=st["position"],
                        inv_freq=st["inv_freq"], interleaved=st["case"]["interleaved"], q=st["q"], q_out=st["q_out"])
        return q, st["k_pages"], st["v_pages"]
    return beam.attend(st["q"], st["k_pages"], st["v_pages"], st["table"], st["prefix"], st["tree"], st["mask"], max_len=st["max_len"],
                       return_lse=True)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _exact_select(st):
    c = st["case"]
    V, m = c["V"], c["k_out"]
    token, back = np.full((c["B"], m), PAD, np.int32), np.full((c["B"], m), -1, np.int32)
    score, out = np.full((c["B"], m), -np.inf), np.full((c["B"], m), DEAD, np.uint8)
    flags, parent = st["flags"].cpu().numpy(), st["score"].double()
    for b in range(c["B"]):
        s = torch.log_softmax(st["logits"][b].double(), dim=1) + parent[b][:, None]
        for h in range(c["k"]):
            if flags[b, h]:
                s[h] = -math.inf
                if flags[b, h] & FINISHED:
                    s[h, PAD] = parent[b, h]
        s = s.flatten()
        at = torch.nonzero(s >= torch.kthvalue(s, s.numel() - m + 1).values).flatten()
        val, at = s[at].cpu().numpy(), at.cpu().numpy()
        order = np.lexsort((at, -val))[:m]
        order = order[val[order] > -np.inf]
        f = len(order)
        score[b, :f], token[b, :f], back[b, :f] = val[order], at[order] % V, at[order] // V
        out[b, :f] = [FINISHED if w == EOS or flags[b, h] else 0 for h, w in zip(back[b, :f], token[b, :f])]
    return token, back, score, out


def _exact_reorder(st):
    outs = []
    back = st["back"].cpu().numpy()
    for s in st["src"]:
        o = torch.zeros(s.shape, dtype=torch.float64, device=s.device)
        for b in range(back.shape[0]):
            for h in range(back.shape[1]):
                if back[b, h] >= 0:
                    o[b, h] = s[b, back[b, h]]
        outs.append(o)
    return outs


def _exact_append(st):
    c = st["case"]
    rot, page = c["rot"], c["page"]
    q_out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
    first, table = st["first"].tolist(), st["table"].tolist()
    pairs = torch.arange(rot // 2, device=q_out.device)
    lo, hi = (2 * pairs, 2 * pairs + 1) if c["interleaved"] else (pairs, pairs + rot // 2)
    for b in range(c["B"]):
        n = c["n"] if st["count"] is None else st["count"].tolist()[b]
        pos = torch.arange(first[b], first[b] + n, device=q_out.device) if st["position"] is None else st["position"][b]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=q_out.device), pos.double()[:, None] * st["inv_freq"].double())[:, None]

        def rotate(x):
            y = x[:n].double()
            z = torch.complex(y[..., lo], y[..., hi]) * turn
            y[..., lo], y[..., hi] = z.real, z.imag
            return y

        q_out[b, :n] = rotate(st["q"][b])
        at = np.arange(first[b], first[b] + n)
        page_of = torch.tensor([table[b][p] for p in at // page], device=q_out.device)
        k_pages[page_of, torch.from_numpy(at % page).to(q_out.device)] = rotate(st["k"][b])
        v_pages[page_of, torch.from_numpy(at % page).to(q_out.device)] = st["v"][b, :n].double()
    return q_out, k_pages, v_pages


def _exact_attend(st):
    c = st["case"]
    n, Hq, G = c["n"], c["Hq"], c["Hq"] // c["Hkv"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    lse = torch.full(st["q"].shape[:3], -math.inf, dtype=torch.float64, device=out.device)
    prefix, tree = st["prefix"].tolist(), st["tree"].tolist()
    words = None if st["mask"] is None else st["mask"].cpu().numpy().view(np.uint64)
    for b in range(c["B"]):
        L = prefix[b] + tree[b]
        seen = np.ones((n, L), bool)
        if words is None:
            seen[:, prefix[b]:] = np.tri(n, tree[b], tree[b] - n, dtype=bool)
        else:
            bits = np.unpackbits(words[b].view(np.uint8), axis=1, bitorder="little")
            seen[:, prefix[b]:] = bits[:, :tree[b]].astype(bool)
        hidden = torch.from_numpy(~seen).to(out.device)
        pages = st["table"][b, :-(-L // c["page"])].long()
        for h in range(c["Hkv"]):
            k = st["k_pages"][pages, :, h].reshape(-1, c["D"])[:L].double()
            v = st["v_pages"][pages, :, h].reshape(-1, c["D"])[:L].double()
            for r in range(h * G, h * G + G):
                s = (st["q"][b, :, r].double() @ k.t() / math.sqrt(c["D"])).masked_fill(hidden, -math.inf)
                lse[b, :, r] = torch.logsumexp(s, dim=1)
                out[b, :, r] = torch.nan_to_num((s - lse[b, :, r, None]).exp()) @ v
    return out, lse


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "reorder" and case["B"] * case["k"] * case["states"] > 200000:
        return None
    return {"select": _exact_select, "reorder": _exact_reorder, "append": _exact_append, "attend": _exact_attend}[case["op"]](st)
