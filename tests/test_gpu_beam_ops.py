"""-m gpu: the operators of include/dba_beam.h against plain statements in 64 bits.

Tolerances.  u is half a step of the result's type (2^-24, 2^-11, 2^-8 of the value).
  selection   the score is rounded once (u) behind a normaliser whose exponentials are off by 2^-22 of themselves at most
              (argument and result of an fp32 exp2): |s| u + 2^-22.  Tokens and back-pointers are equal, as the inputs leave gaps.
  append      one rounding (u |y|) behind an fp32 rotation: cos and sin to 4 u32, two products and a sum: 8 u32 (|x0| + |x1|).
  attention   with A = sum_t p_t |v_t|: weights rounded to the type (u A) and the result (u |o|); a score is a sum of D products
              in fp32, off by e = (D + 8) u32 sum |q k| scale, so a weight by 2 e and the exponential's 2^-21; sums over L tokens
              in fp32: L u32 A.  The normaliser: e + 2^-21 + L u32.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.float16, torch.bfloat16]
EOS, PAD = 2, 0


@pytest.fixture(scope="module")
def beam():
    from paper_1804_06609_amd import beam as m
    m.load()
    return m


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- selection -------------------------------------------------------------------------------------------------------
def plain_select(logits, score, flags, k_out):
    """On the CPU in 64 bits, a sort of everything."""
    B, k, V = logits.shape
    x = logits.double().numpy()
    token, back = np.full((B, k_out), PAD, np.int32), np.full((B, k_out), -1, np.int32)
    out, fl = np.full((B, k_out), -np.inf), np.full((B, k_out), 2, np.uint8)
    for b in range(B):
        s = np.full((k, V), -np.inf)
        for h in range(k):
            sc = float(score[b, h])
            f = 0 if flags is None else int(flags[b, h])
            if (f & 2) or not math.isfinite(sc):
                continue
            if f & 1:
                s[h, PAD] = sc
                continue
            with np.errstate(all="ignore"):
                top = x[b, h].max()
                total = np.exp(x[b, h] - top).sum()
            if math.isfinite(top) and math.isfinite(total):
                s[h] = sc + ((x[b, h] - top) - math.log(total))
        s = s.reshape(-1)
        order = np.lexsort((np.arange(k * V), -s))[:k_out]
        order = order[s[order] > -np.inf]
        for i, at in enumerate(order):
            back[b, i], token[b, i], out[b, i] = at // V, at % V, s[at]
            fl[b, i] = 1 if token[b, i] == EOS or (flags is not None and int(flags[b, at // V]) & 1) else 0
    return token, back, out, fl


def check_select(beam, logits, score, flags, k_out, logits_dev=None):
    dev = logits.cuda() if logits_dev is None else logits_dev
    got = beam.select(dev, score.cuda(), None if flags is None else flags.cuda(), k_out, EOS, PAD)
    token, back, out, fl = plain_select(logits, score, flags, k_out)
    g = [x.cpu().numpy() for x in got]
    assert np.array_equal(g[1], back) and np.array_equal(g[0], token) and np.array_equal(g[3], fl)
    assert np.array_equal(np.isfinite(g[2]), np.isfinite(out)) and np.array_equal(g[2][~np.isfinite(out)], out[~np.isfinite(out)])
    f = np.isfinite(out)
    assert (np.abs(g[2][f] - out[f]) <= np.abs(out[f]) * U32 + 2.0 ** -22).all()


def a_beam(seed, B, k, V, dtype):
    g = gen(seed)
    logits = (torch.randn(B, k, V, generator=g) * 2).to(dtype)
    score = -torch.rand(B, k, generator=g) * 4 - 5
    flags = (torch.rand(B, k, generator=g) < 0.15).to(torch.uint8)
    return logits, score, flags


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,k,k_out,V", [(1, 1, 1, 3), (1, 1, 1, 1025), (2, 5, 5, 1000), (1, 1, 10, 32000), (3, 7, 7, 50001), (2, 20, 40, 8191), (2, 64, 64, 8193),
                                         (1, 3, 64, 100003), (5, 64, 1, 17), (2, 4, 64, 9)])
def test_select(beam, dtype, B, k, k_out, V):
    logits, score, flags = a_beam(B * 1000 + V, B, k, V, dtype)
    check_select(beam, logits, score, flags, k_out)
    check_select(beam, logits, score, None, k_out)


@pytest.mark.parametrize("dtype", TYPES)
def test_select_from_strided_logits(beam, dtype):
    logits, score, flags = a_beam(3, 3, 6, 777, dtype)
    for lead, ld in ((0, 777), (1, 779), (3, 1000)):
        room = torch.full((3, 6, 2, ld + lead), float("nan"), dtype=dtype)
        room[:, :, 1, lead:lead + 777] = logits
        check_select(beam, logits, score, flags, 6, room.cuda()[:, :, 1, lead:lead + 777])


@pytest.mark.parametrize("dtype", TYPES)
def test_select_masks_and_values_that_are_not_finite(beam, dtype):
    logits, score, flags = a_beam(4, 8, 6, 5000, dtype)
    low = torch.finfo(dtype).min
    logits[0, :, 100:] = -math.inf                     # few tokens are left
    logits[1, :, 2:] = low                             # the same with the type's lowest value
    logits[2] = -math.inf                              # nothing is left: an empty beam
    logits[3, 1] = low                                 # a row of lowest values is a uniform row
    logits[4, 0, 77] = math.nan
    logits[4, 1, 78] = math.inf
    logits[4, 2, :] = -math.inf
    logits[5, 0] = math.nan                            # rows that are not looked at
    flags[5, 0], flags[5, 1] = 2, 1
    logits[5, 1] = math.inf
    score[6, :] = -math.inf
    score[6, 3], score[6, 4], score[6, 5] = -1.0, math.nan, math.inf
    flags[6] = 0
    logits[7, :, ::2] = -math.inf
    check_select(beam, logits, score, flags, 6)
    check_select(beam, logits, score, flags, 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [100, 5000, 40000])
def test_select_equal_logits_go_to_the_first(beam, dtype, V):
    logits = torch.zeros(4, 5, V, dtype=dtype)
    logits[1] = torch.randint(0, 3, (5, V), generator=gen(V)).to(dtype)
    logits[2, :, V // 2:] = -0.0
    logits[3, 2] = -1.0
    score = torch.full((4, 5), -2.0)                   # equal rows, too
    score[1] = torch.tensor([-2.0, -2.5, -2.25, -3.0, -9.0])
    for k_out in (1, 33, 64):
        got = beam.select(logits.cuda(), score.cuda(), None, k_out, EOS, PAD)
        for b in (0, 2):
            n = min(k_out, V)
            assert got[0][b, :n].tolist() == list(range(n)) and got[1][b, :n].tolist() == [0] * n
        token, back, out, fl = plain_select(logits[1:2], score[1:2], None, k_out)
        assert got[0][1].tolist() == token[0].tolist() and got[1][1].tolist() == back[0].tolist()


@pytest.mark.parametrize("dtype", TYPES)
def test_select_where_more_reach_the_bound_than_there_is_room_for(beam, dtype):
    """Fewer lists than slots, so that every list's keys are looked at; and thousands of equal scores, of which the first count."""
    logits, score, flags = a_beam(6, 2, 28, 22357, dtype)
    check_select(beam, logits, score, None, 62)
    logits = torch.zeros(2, 20, 40000, dtype=dtype)
    logits[1, :, :100] = -1
    score = torch.full((2, 20), -2.0)
    score[1, :5] = -3.0                                # the sixth row's tokens from the hundredth on
    got = [x.cpu() for x in beam.select(logits.cuda(), score.cuda(), None, 64, EOS, PAD)]
    assert got[0][0].tolist() == list(range(64)) and got[1][0].tolist() == [0] * 64
    assert got[0][1].tolist() == list(range(100, 164)) and got[1][1].tolist() == [5] * 64


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [200, 1164, 20000, 70001])
def test_select_where_the_best_lie_together(beam, dtype, V):
    """Tokens in the order of their frequency, up and down; coarse logits, of which many are equal; a block of tokens allowed."""
    g = gen(V)
    x = torch.randn(4, 9, V, generator=g) * 2
    x[0] = x[0].sort(dim=1, descending=True).values
    x[1] = x[1].sort(dim=1).values
    x[2] = (x[2] * 2).round() / 2
    x[3, :, V // 2:] = -math.inf
    score = -torch.rand(4, 9, generator=g) * 4 - 5
    for k_out in (1, 9, 31, 64):
        check_select(beam, x.to(dtype), score, None, k_out)


def test_select_twice_is_the_same(beam):
    logits, score, flags = a_beam(9, 4, 20, 32000, torch.float32)
    args = [logits.cuda(), score.cuda(), flags.cuda(), 20, EOS, PAD]
    first = [x.cpu() for x in beam.select(*args)]
    for _ in range(3):
        assert all(torch.equal(a, b.cpu()) for a, b in zip(first, beam.select(*args)))


# ---- reordering ------------------------------------------------------------------------------------------------------
def plain_reorder(back, x):
    out = torch.zeros_like(x)
    for b in range(back.shape[0]):
        for h in range(back.shape[1]):
            if 0 <= back[b, h] < back.shape[1]:
                out[b, h] = x[b, back[b, h]]
    return out


def some_states(seed, B, k):
    g = gen(seed)
    r = lambda *s: torch.randint(-100, 100, (B, k) + s, generator=g)
    return [r(512).float(), r(3).to(torch.int8), r(7, 5).to(torch.bfloat16), r(2).long(), r(4, 10, 8).half(), r().int(), r(6).to(torch.int16)]


@pytest.mark.parametrize("B,k", [(1, 1), (1, 5), (3, 8), (2, 16), (2, 20), (4, 33), (1, 64)])
def test_reorder(beam, B, k):
    back = torch.randint(-1, k, (B, k), generator=gen(k), dtype=torch.int32)
    back[0, 0] = k - 1
    if k > 4:
        back[0, 1], back[0, 2], back[0, 3] = k, -2**31, 2**31 - 1        # as good as none
    states = some_states(7, B, k)
    want = [plain_reorder(back, s) for s in states]
    dev = [s.cuda() for s in states]
    out = [torch.full_like(d, 9) for d in dev]
    assert beam.reorder(back.cuda(), dev, out) is out
    for s, d, o, w in zip(states, dev, out, want):
        assert torch.equal(d.cpu(), s) and torch.equal(o.cpu(), w)
    beam.reorder(back.cuda(), dev)                                       # in place
    for d, w in zip(dev, want):
        assert torch.equal(d.cpu(), w)


def test_reorder_of_the_places_in_use(beam):
    x = torch.randn(3, 6, 4, 11, 8, generator=gen(1)).half()
    back = torch.randint(0, 6, (3, 6), generator=gen(2), dtype=torch.int32)
    dev = x.cuda()
    beam.reorder(back.cuda(), [dev[:, :, :, :7]])
    want = x.clone()
    want[:, :, :, :7] = plain_reorder(back, x[:, :, :, :7])
    assert torch.equal(dev.cpu(), want)
    dense = torch.zeros(3, 6, 4, 7, 8, dtype=torch.float16, device="cuda")   # a dense buffer for pieces of a larger one
    beam.reorder(back.cuda(), [x.cuda()[:, :, :, :7]], [dense])
    assert torch.equal(dense.cpu(), want[:, :, :, :7])
    beam.reorder(back.cuda(), [x.cuda()[:, :, :, :0]], [dense[:, :, :, :0]])


def test_reorder_of_more_states_than_one_launch_takes(beam):
    xs = [torch.randn(2, 4, 3 + i, generator=gen(i)) for i in range(60)]
    back = torch.tensor([[1, 1, -1, 2], [3, 2, 1, 0]], dtype=torch.int32)
    dev = [x.cuda() for x in xs]
    beam.reorder(back.cuda(), dev)
    for x, d in zip(xs, dev):
        assert torch.equal(d.cpu(), plain_reorder(back, x))


def test_reorder_of_no_rows_is_refused(beam):
    from paper_1804_06609_amd import DbaError
    for shape in ((0, 4), (3, 0)):
        with pytest.raises(DbaError, match="B"):
            beam.reorder(torch.zeros(shape, dtype=torch.int32, device="cuda"), [torch.zeros(shape + (5,), device="cuda")])


# ---- caches ------------------------------------------------------------------------------------------------------------
def a_cache(seed, B, tokens, heads, D, page, dtype, layout="nhd", fill=None):
    """Pages of B sentences in random order; "hnd" has the heads before the tokens of a page."""
    per = -(-tokens // page)
    n = B * per + 2
    g = gen(seed)
    shape = (n, page, heads, D) if layout == "nhd" else (n, heads, page, D)
    k, v = (torch.randn(shape, generator=g) if fill is None else torch.full(shape, fill) for _ in range(2))
    k, v = k.to(dtype).cuda(), v.to(dtype).cuda()
    if layout == "hnd":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    table = torch.randperm(n, generator=g)[:B * per].reshape(B, per).int()
    return k, v, table


def rows_of(pages, table, b, tokens):
    """[tokens, heads, D] of a sentence, on the CPU in 64 bits."""
    p, page = pages.cpu().double(), pages.shape[1]
    return torch.stack([p[table[b, t // page], t % page] for t in range(tokens)]) if tokens else p[0, :0]


def rotated(x, position, inv_freq, interleaved):
    """x [n, heads, D] in 64 bits and what an fp32 rotation may be off by."""
    r = inv_freq.numel()
    a = position.double()[:, None] * inv_freq.double()
    c, s = a.cos()[:, None], a.sin()[:, None]
    y, tol = x.clone(), torch.zeros_like(x)
    lo = torch.arange(r) * 2 if interleaved else torch.arange(r)
    hi = lo + 1 if interleaved else lo + r
    y[..., lo], y[..., hi] = x[..., lo] * c - x[..., hi] * s, x[..., hi] * c + x[..., lo] * s
    tol[..., lo] = tol[..., hi] = 8 * U32 * (x[..., lo].abs() + x[..., hi].abs())
    return y, tol


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,n,Hq,Hkv,D,rot,page,layout", [
    (1, 1, 1, 1, 8, 0, 1, "nhd"), (2, 5, 4, 4, 64, 64, 16, "nhd"), (3, 17, 6, 2, 80, 48, 8, "hnd"), (2, 33, 8, 1, 256, 256, 32, "nhd"),
    (2, 70, 4, 4, 128, 64, 64, "hnd"), (1, 3, 9, 3, 96, 96, 2, "nhd"), (2, 4, 2, 2, 24, 16, 4, "nhd")])
def test_append(beam, dtype, interleaved, B, n, Hq, Hkv, D, rot, page, layout):
    g = gen(n * D)
    cap = 3 * page + n
    k_pages, v_pages, table = a_cache(5, B, cap, Hkv, D, page, dtype, layout, fill=7.0)
    k, v, q = (torch.randn(B, n, h, D, generator=g).to(dtype) for h in (Hkv, Hkv, Hq))
    first = torch.randint(0, 3 * page, (B,), generator=g).int()
    inv = (10000.0 ** (-torch.arange(0, rot, 2).double() / max(rot, 1))).float()
    for position, count in ((None, None), (torch.randint(-5, 2**20, (B, n), generator=g).int(), torch.randint(0, n + 2, (B,), generator=g).int())):
        kp, vp = k_pages.clone(), v_pages.clone()
        q_dev = q.cuda()
        q_out = beam.append(k.cuda(), v.cuda(), kp, vp, table.cuda(), first.cuda(), None if count is None else count.cuda(),
                            position=None if position is None else position.cuda(), inv_freq=inv.cuda() if rot else None,
                            interleaved=interleaved, q=q_dev)
        beam.append(k.cuda(), v.cuda(), kp, vp, table.cuda(), first.cuda(), None if count is None else count.cuda(),
                    position=None if position is None else position.cuda(), inv_freq=inv.cuda() if rot else None,
                    interleaved=interleaved, q=q_dev, q_out=q_dev)
        assert torch.equal(q_dev, q_out)                                 # in place, too
        kc, vc = kp.cpu().double(), vp.cpu().double()
        touched = torch.zeros(kc.shape[:2], dtype=torch.bool)
        for b in range(B):
            m = n if count is None else min(n, int(count[b]))
            pos = first[b] + torch.arange(n) if position is None else position[b]
            want_k, tol_k = rotated(k[b].double(), pos, inv, interleaved)
            want_q, tol_q = rotated(q[b].double(), pos, inv, interleaved)
            for i in range(m):
                t = int(first[b]) + i
                at = table[b, t // page], t % page
                touched[at] = True
                assert ((kc[at] - want_k[i]).abs() <= U[dtype] * want_k[i].abs() + tol_k[i] * (1 + U[dtype])).all()
                assert torch.equal(vc[at], v[b, i].double())
            got = q_out[b].cpu().double()
            assert ((got[:m] - want_q[:m]).abs() <= U[dtype] * want_q[:m].abs() + tol_q[:m] * (1 + U[dtype])).all()
            assert (got[m:] == 0).all()
        assert (kc[~touched] == 7).all() and (vc[~touched] == 7).all()   # nothing else was written


def test_append_into_pages_that_are_not_there(beam):
    k_pages, v_pages, table = a_cache(1, 2, 32, 2, 16, 4, torch.float16, fill=7.0)
    table[0, 2], table[1, 0], table[1, 3] = -1, 2**31 - 1, -2**31
    k = torch.randn(2, 40, 2, 16, generator=gen(1)).half()               # more than the table has room for
    first = torch.tensor([-3, 4], dtype=torch.int32)
    beam.append(k.cuda(), k.cuda(), k_pages, v_pages, table.cuda(), first.cuda())
    got, touched = v_pages.cpu(), torch.zeros(v_pages.shape[:2], dtype=torch.bool)
    for b in range(2):
        for i in range(40):
            t = int(first[b]) + i
            if 0 <= t < 32 and 0 <= table[b, t // 4] < len(k_pages):
                at = int(table[b, t // 4]), t % 4
                touched[at] = True
                assert torch.equal(got[at], k[b, i])
    assert (got[~touched] == 7).all() and (k_pages.cpu()[~touched] == 7).all()


def test_append_of_parts_of_a_fused_projection(beam):
    k_pages, v_pages, table = a_cache(1, 2, 32, 2, 64, 8, torch.bfloat16)
    qkv = torch.randn(2, 6, 8, 64, generator=gen(4)).bfloat16().cuda()
    first = torch.tensor([0, 9], dtype=torch.int32).cuda()
    inv = torch.rand(32, generator=gen(5)).cuda()
    ref = [k_pages.clone(), v_pages.clone()]
    q = beam.append(qkv[:, :, 4:6], qkv[:, :, 6:], k_pages, v_pages, table.cuda(), first, inv_freq=inv, q=qkv[:, :, :4])
    q2 = beam.append(qkv[:, :, 4:6].contiguous(), qkv[:, :, 6:].contiguous(), ref[0], ref[1], table.cuda(), first, inv_freq=inv, q=qkv[:, :, :4].contiguous())
    assert torch.equal(q, q2) and torch.equal(k_pages, ref[0]) and torch.equal(v_pages, ref[1])


# ---- attention ---------------------------------------------------------------------------------------------------------
def plain_attend(q, k_pages, v_pages, table, prefix, tree, seen_of_tree, scale):
    """seen_of_tree(b, i, j) -> bool.  Returns out, lse and what each may be off by, in 64 bits, from a loop over sentences and heads."""
    B, n, Hq, D = q.shape
    page, Hkv = k_pages.shape[1], k_pages.shape[2]
    out, tol = torch.zeros(B, n, Hq, D, dtype=torch.float64), torch.zeros(B, n, Hq, D, dtype=torch.float64)
    lse, lse_tol = torch.full((B, n, Hq), -math.inf, dtype=torch.float64), torch.zeros(B, n, Hq, dtype=torch.float64)
    kp, vp = k_pages.cpu().double(), v_pages.cpu().double()
    u = U[q.dtype]
    for b in range(B):
        P, T = max(0, int(prefix[b])), max(0, int(tree[b]))
        L = min(P + T, table.shape[1] * page)
        toks = [t for t in range(L) if 0 <= table[b, t // page] < len(kp)]
        if not toks:
            continue
        at = torch.tensor([int(table[b, t // page]) * page + t % page for t in toks])
        k, v = kp.reshape(-1, Hkv, D)[at], vp.reshape(-1, Hkv, D)[at]
        see = torch.tensor([[t < P or bool(seen_of_tree(b, i, t - P)) for t in toks] for i in range(n)])
        for i in range(n):
            m = see[i].nonzero().flatten()
            if not len(m):
                continue
            for h in range(Hq):
                kk, vv = k[m, h * Hkv // Hq], v[m, h * Hkv // Hq]
                x = q[b, i, h].cpu().double()
                s = kk @ x * scale
                lse[b, i, h] = torch.logsumexp(s, 0)
                p = (s - lse[b, i, h]).exp()
                out[b, i, h] = p @ vv
                e = (D + 8) * U32 * float((kk.abs() @ x.abs()).max()) * abs(scale)
                tol[b, i, h] = u * out[b, i, h].abs() + (p @ vv.abs()) * (u + 2 * (2 * e + 2.0 ** -21) + len(m) * U32)
                lse_tol[b, i, h] = 2 * e + 2.0 ** -20 + len(m) * U32 + U32 * abs(float(lse[b, i, h]))
    return out, lse, tol, lse_tol


def near(got, lse, want):
    o, l, tol, ltol = want
    g = got.cpu().double()
    assert torch.isfinite(g).all()
    assert ((g - o).abs() <= tol).all(), float(((g - o).abs() - tol).max())
    e = lse.cpu().double()
    dead = l == -math.inf
    assert torch.equal(e == -math.inf, dead) and not torch.isnan(e).any()
    assert ((e - l).abs()[~dead] <= ltol[~dead]).all(), float(((e - l).abs() - ltol)[~dead].max())


def random_mask(seed, B, n, words, density=0.5):
    bits = np.random.RandomState(seed).rand(B, n, words * 64) < density
    packed = np.packbits(bits, axis=2, bitorder="little").view(np.int64).reshape(B, n, words)
    return torch.from_numpy(packed.copy()), bits


def check_attend(beam, dtype, B, n, Hq, Hkv, D, page, prefix, tree, masked, layout="nhd", seed=0, scale=None, density=0.5, max_len=None):
    prefix, tree = torch.tensor(prefix, dtype=torch.int32), torch.tensor(tree, dtype=torch.int32)
    cap = max(1, int((prefix.clamp(min=0) + tree.clamp(min=0)).max()))
    k_pages, v_pages, table = a_cache(seed, B, cap, Hkv, D, page, dtype, layout)
    q = torch.randn(B, n, Hq, D, generator=gen(seed + 1)).to(dtype).cuda()
    words = -(-max(1, int(tree.max())) // 64)
    mask = bits = None
    if masked:
        mask, bits = random_mask(seed, B, n, words, density)
        seen = lambda b, i, j: bits[b, i, j]
    else:
        seen = lambda b, i, j: j <= int(tree[b]) - n + i
    got, lse = beam.attend(q, k_pages, v_pages, table.cuda(), prefix.cuda(), tree.cuda(), mask.cuda() if masked else None, scale=scale,
                           max_len=max_len, return_lse=True)
    near(got, lse, plain_attend(q, k_pages, v_pages, table, prefix, tree, seen, D ** -0.5 if scale is None else scale))


SHAPES = [
    # B, n, Hq, Hkv, D, page, prefix, tree
    (1, 1, 1, 1, 8, 1, [1], [0]),
    (1, 1, 8, 8, 64, 16, [1000], [1]),
    (3, 5, 4, 4, 64, 16, [0, 17, 130], [70, 64, 5]),
    (2, 20, 8, 2, 128, 16, [63, 65], [100, 40]),
    (2, 7, 6, 2, 80, 8, [200, 3], [33, 130]),
    (2, 3, 16, 1, 96, 32, [31, 500], [1, 63]),
    (1, 33, 8, 8, 32, 64, [77], [129]),
    (2, 2, 6, 3, 256, 4, [100, 5], [65, 20]),
    (1, 63, 16, 2, 128, 16, [700], [63]),
    (4, 1, 3, 1, 24, 2, [0, 1, 2, 3], [1, 0, 2, 1]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_attend_with_a_mask(beam, dtype, shape):
    check_attend(beam, dtype, *shape, masked=True, seed=len(shape[6]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_attend_along_a_chain(beam, dtype, shape):
    check_attend(beam, dtype, *shape, masked=False, layout="hnd", seed=3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [150, 300])
def test_attend_of_a_prompt(beam, dtype, n):
    check_attend(beam, dtype, 2, n, 4, 2, 64, 16, [0, 37], [n, n], masked=False)


@pytest.mark.parametrize("dtype", TYPES)
def test_attend_over_many_tokens(beam, dtype):
    check_attend(beam, dtype, 1, 3, 4, 2, 64, 64, [9000], [50], masked=True)
    check_attend(beam, dtype, 2, 1, 8, 1, 128, 16, [3001, 17], [1, 0], masked=False)


@pytest.mark.parametrize("dtype", TYPES)
def test_attend_nodes_that_see_nothing(beam, dtype):
    check_attend(beam, dtype, 3, 6, 4, 2, 64, 8, [0, 0, -5], [100, 0, 10], masked=True, density=0.02)
    check_attend(beam, dtype, 3, 6, 4, 2, 64, 8, [0, 0, 3], [2, 0, -7], masked=False)
    q = torch.randn(1, 4, 2, 32).to(dtype).cuda()
    k_pages, v_pages, table = a_cache(1, 1, 64, 2, 32, 16, dtype)
    one = torch.ones(1, dtype=torch.int32).cuda()
    out, lse = beam.attend(q, k_pages, v_pages, table.cuda(), one * 0, one * 64, torch.zeros(1, 4, 0, dtype=torch.int64).cuda(), return_lse=True)
    assert (out == 0).all() and (lse == -math.inf).all()
    out, lse = beam.attend(q, k_pages, v_pages, table.cuda(), one * 0, None, return_lse=True)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_attend_with_large_scores(beam, dtype):
    check_attend(beam, dtype, 2, 5, 4, 2, 64, 16, [300, 20], [40, 64], masked=True, scale=3.0)
    check_attend(beam, dtype, 2, 5, 4, 2, 64, 16, [300, 20], [40, 64], masked=True, scale=-0.5)
    check_attend(beam, dtype, 2, 5, 4, 2, 64, 16, [300, 20], [40, 64], masked=True, scale=0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_attend_what_is_not_seen_does_not_matter(beam, dtype, bad):
    """Behind the end, in pages that are not there, and in tokens that some nodes see and others do not."""
    B, n, H, D, page = 2, 20, 2, 64, 8
    prefix, tree = torch.tensor([70, 9], dtype=torch.int32), torch.tensor([90, 41], dtype=torch.int32)
    k_pages, v_pages, table = a_cache(2, B, 200, H, D, page, dtype)
    q = torch.randn(B, n, 2 * H, D, generator=gen(3)).to(dtype).cuda()
    mask, bits = random_mask(1, B, n, 2)
    bits[:, n // 2:, 30], bits[:, :n // 2, 30] = True, False             # node by node
    bits[:, :, 31] = False                                              # nobody sees it
    mask = torch.from_numpy(np.packbits(bits, axis=2, bitorder="little").view(np.int64).reshape(B, n, 2).copy())
    table[0, 3] = -1
    seen = lambda b, i, j: bits[b, i, j]
    want = plain_attend(q, k_pages, v_pages, table, prefix, tree, seen, D ** -0.5)
    kd, vd = k_pages.clone(), v_pages.clone()
    for b in range(B):
        end = int(prefix[b] + tree[b])
        spoil = [int(prefix[b]) + 31] + list(range(end, table.shape[1] * page))
        for t in spoil:
            if 0 <= table[b, t // page]:
                kd[table[b, t // page], t % page] = bad
                vd[table[b, t // page], t % page] = bad
    got, lse = beam.attend(q, kd, vd, table.cuda(), prefix.cuda(), tree.cuda(), mask.cuda(), return_lse=True)
    near(got, lse, want)
    for b in range(B):                                                  # now token 30 as well: the first half of the nodes does not see it
        t = int(prefix[b]) + 30
        kd[table[b, t // page], t % page] = bad
        vd[table[b, t // page], t % page] = bad
    got, lse = beam.attend(q, kd, vd, table.cuda(), prefix.cuda(), tree.cuda(), mask.cuda(), return_lse=True)
    half = [x[:, :n // 2] for x in want]
    near(got[:, :n // 2], lse[:, :n // 2], half)
    if bad != -math.inf:                                                # who does see it is told
        assert not torch.isfinite(got[:, n // 2:].float()).all(dim=3).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 70])
def test_attend_over_a_long_tail_of_small_weights(beam, dtype, n):
    """One token of weight 1 whose value is 0, thousands of 2^-26 with values of 1: the output is theirs alone."""
    D, L = 8, 6000
    k_pages, v_pages, table = a_cache(4, 1, L, 1, D, 16, dtype, fill=0.0)
    v_pages[...] = 1
    at = int(table[0, 1]), 3
    k_pages[at] = 0
    k_pages[at[0], at[1], 0, 0] = 18.0
    v_pages[at] = 0
    q = torch.zeros(1, n, 1, D, dtype=dtype, device="cuda")
    q[..., 0] = 1
    prefix, none = torch.tensor([L], dtype=torch.int32), torch.tensor([0], dtype=torch.int32)
    got, lse = beam.attend(q, k_pages, v_pages, table.cuda(), prefix.cuda(), scale=1.0, return_lse=True)
    near(got, lse, plain_attend(q, k_pages, v_pages, table, prefix, none, None, 1.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,n,Hq,Hkv,D,masked", [(128, 2, 16, 8, 64, True), (128, 1, 8, 8, 128, False), (64, 20, 16, 16, 24, True), (52, 3, 20, 20, 80, True), (32, 2, 16, 16, 256, False),
                                                 (128, 9, 32, 8, 64, True)])
def test_attend_of_many_sentences(beam, dtype, B, n, Hq, Hkv, D, masked):
    r = np.random.RandomState(B + D)
    prefix, tree = r.randint(0, 40, B), r.randint(0, 70, B)
    prefix[0], tree[0] = 150, 64
    prefix[1], tree[1] = 0, 0
    check_attend(beam, dtype, B, n, Hq, Hkv, D, 8, prefix.tolist(), tree.tolist(), masked=masked, seed=5, density=0.2)


@pytest.mark.parametrize("dtype", TYPES)
def test_attend_of_many_sentences_what_is_not_seen_does_not_matter(beam, dtype):
    B, n, H, D, page = 128, 2, 8, 64, 8
    prefix, tree = torch.full((B,), 5, dtype=torch.int32), torch.full((B,), 33, dtype=torch.int32)
    k_pages, v_pages, table = a_cache(2, B, 40, H, D, page, dtype)
    q = torch.randn(B, n, H, D, generator=gen(3)).to(dtype).cuda()
    mask, bits = random_mask(1, B, n, 1)
    bits[:, 0, 30], bits[:, 1, 30] = False, True
    mask = torch.from_numpy(np.packbits(bits, axis=2, bitorder="little").view(np.int64).reshape(B, n, 1).copy())
    want = plain_attend(q, k_pages, v_pages, table, prefix, tree, lambda b, i, j: bits[b, i, j], D ** -0.5)
    at = 5 + 30
    for b in range(B):                                                  # one element of one head is not a number, differently for each sentence
        v_pages[int(table[b, at // page]), at % page, b % H, b % D] = math.nan
    got, lse = beam.attend(q, k_pages, v_pages, table.cuda(), prefix.cuda(), tree.cuda(), mask.cuda(), return_lse=True)
    near(got[:, :1], lse[:, :1], [x[:, :1] for x in want])
    spoiled = torch.zeros(B, H, D, dtype=torch.bool)
    spoiled[torch.arange(B), torch.arange(B) % H, torch.arange(B) % D] = True
    seen = got[:, 1].cpu().double()
    assert torch.equal(torch.isnan(seen), spoiled)
    assert ((seen - want[0][:, 1]).abs()[~spoiled] <= want[2][:, 1][~spoiled]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_attend_no_further_than_max_len(beam, dtype):
    B, n, H, D = 2, 3, 2, 64
    k_pages, v_pages, table = a_cache(2, B, 320, H, D, 16, dtype)
    q = torch.randn(B, n, H, D, generator=gen(3)).to(dtype).cuda()
    prefix, tree = torch.tensor([290, 100], dtype=torch.int32), torch.tensor([30, 60], dtype=torch.int32)
    mask, bits = random_mask(1, B, n, 1)
    for max_len in (1, 100, 131, 300):
        p, t = prefix.clamp(max=max_len), torch.minimum(tree, (max_len - prefix).clamp(min=0))
        got, lse = beam.attend(q, k_pages, v_pages, table.cuda(), prefix.cuda(), tree.cuda(), mask.cuda(), max_len=max_len, return_lse=True)
        near(got, lse, plain_attend(q, k_pages, v_pages, table, p, t, lambda b, i, j: bits[b, i, j], D ** -0.5))


def test_attend_offsets_beyond_32_bits(beam):
    """A pool of 5 GiB: the last pages lie behind 2^31 elements."""
    page, H, D = 1024, 8, 128
    n = (1 << 31) // (page * H * D) + 40
    k_pages = torch.empty((n, page, H, D), dtype=torch.bfloat16, device="cuda")
    v_pages = k_pages                                                    # keys and values may be one tensor
    g = torch.Generator(device="cuda").manual_seed(1)
    last = [n - 1, n - 7, 0]
    for p in last:
        k_pages[p].normal_(generator=g)
    table = torch.tensor([[n - 1, n - 7, 0]], dtype=torch.int32)
    small, t3 = torch.stack([k_pages[p] for p in last]), torch.tensor([[0, 1, 2]], dtype=torch.int32)
    q = torch.randn(1, 2, 8, D, generator=gen(1)).bfloat16().cuda()
    prefix = torch.tensor([2100], dtype=torch.int32).cuda()
    a = beam.attend(q, k_pages, v_pages, table.cuda(), prefix, return_lse=True)
    b = beam.attend(q, small, small, t3.cuda(), prefix, return_lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    x = torch.randn(1, 5, H, D, generator=gen(2)).bfloat16().cuda()
    beam.append(x, x, k_pages, v_pages, table.cuda(), torch.tensor([2040], dtype=torch.int32).cuda())
    assert torch.equal(k_pages[n - 7, 1016:1021], x[0])


# ---- together ----------------------------------------------------------------------------------------------------------
def test_on_a_stream_of_its_own(beam):
    logits, score, flags = a_beam(5, 4, 8, 9000, torch.bfloat16)
    want = plain_select(logits, score, flags, 8)
    dev = [x.cuda() for x in (logits, score, flags)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(5):
            token, back, sc, fl = beam.select(*dev, 8, EOS, PAD)
            state = torch.arange(32, device="cuda", dtype=torch.int32).reshape(4, 8, 1).repeat(1, 1, 1000)
            beam.reorder(back, [state])
    s.synchronize()
    assert np.array_equal(token.cpu().numpy(), want[0]) and np.array_equal(back.cpu().numpy(), want[1])
    rows = torch.from_numpy(want[1]).clamp(min=0) + torch.arange(4)[:, None] * 8
    assert torch.equal(state[:, :, 0].cpu(), torch.where(torch.from_numpy(want[1]) >= 0, rows, 0).int())
    assert torch.equal(state, state[:, :, :1].expand_as(state))


def test_in_a_graph(beam):
    """One time step captured; every replay against the same calls outside, with other work between."""
    B, k, V, H, D, page = 3, 6, 5000, 4, 64, 16
    g = gen(8)
    k_pages, v_pages, table = a_cache(8, B, 200, 2, D, page, torch.bfloat16)
    table = table.cuda()
    first = torch.tensor([10, 100, 55], dtype=torch.int32).cuda()
    tree = torch.full((B,), k, dtype=torch.int32).cuda()
    mask = (torch.ones(1, dtype=torch.int64) << torch.arange(k)).expand(B, k).reshape(B, k, 1).contiguous().cuda()
    x = {n: torch.zeros(B, k, h, D, dtype=torch.bfloat16, device="cuda") for n, h in (("q", H), ("k", 2), ("v", 2))}
    inv = torch.rand(32, generator=g).cuda()
    logits = torch.zeros(B, k, V, device="cuda")
    score = torch.zeros(B, k, device="cuda")

    def step():
        q = beam.append(x["k"], x["v"], k_pages, v_pages, table, first, inv_freq=inv, q=x["q"])
        o, lse = beam.attend(q, k_pages, v_pages, table, first, tree, mask, return_lse=True)
        picked = beam.select(logits, score, None, k, EOS, PAD)
        moved = o.clone()
        beam.reorder(picked[1], [moved])
        return (o, lse, moved) + picked

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        for t in x.values():
            t.copy_(torch.randn(t.shape, generator=g))
        logits.copy_(torch.randn(logits.shape, generator=g))
        score.copy_(-torch.rand(score.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
