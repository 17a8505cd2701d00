"""-m gpu: appending with norms and several axes, attention behind a common prefix, weighing and eviction of cached tokens, against plain statements in 64 bits.

Tolerances.  u is half a step of the result's type (2^-24, 2^-11, 2^-8 of the value), u32 that of fp32.
  append      squares are added up in fp32, eight in a row at most, then over two such rows and 32 lanes, and the mean is one more step: 15 u32 of
              it, half of which its root has; the root's reciprocal is good to a step (2 u32), and two products follow: 12 u32 |y|; the rotation of those
              8 u32 (|y0| + |y1|) as without norms, and one rounding: u |z|, or half a step of the type's subnormals: below 2^-14 fp16 has steps of
              2^-24 whatever the value (e.g. -2.0894e-05 is rounded by 2.70e-08, which is more than 2^-11 of it and less than 2^-25).
  shared      as attention in test_gpu_beam_ops.py, over all tokens of both kinds; the join adds one fp32 product and sum a part, which L u32 A holds.
  weigh       a weight is exp(x - lse): x is off by e = (D + 8) u32 sum |q k| scale, the argument of the exponential by 4 u32 (|x| + |lse|) more, its result
              by 2^-21 of itself; a sum of R weights by R u32 of itself, and of sum and score by u32.
  evict       nothing is computed: equal.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_beam_ops import TYPES, U, U32, a_cache, beam, gen, near, random_mask  # noqa: F401

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf
LEAST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def cuda(*x):
    return [None if t is None else t.cuda() for t in x]


# ---- appending -------------------------------------------------------------------------------------------------------
def normed_rotated(x, weight, eps, position, axis, inv_freq, interleaved):
    """x [n, heads, D], position [n, pairs' axes]: (result, what it may be off by), in 64 bits."""
    y, tol = x.double(), torch.zeros_like(x, dtype=torch.float64)
    if eps is not None:
        y = y / (y.square().mean(dim=-1, keepdim=True) + eps).sqrt() * (1.0 if weight is None else weight.double())
        tol = 12 * U32 * y.abs()
    r = len(inv_freq)
    if axis is not None:
        pos = torch.stack([position[:, a] if 0 <= a < position.shape[1] else torch.zeros(len(x)) for a in axis.tolist()], dim=1).double()
    else:
        pos = position.double()[:, None]
    a = pos * inv_freq.double()
    c, s = a.cos()[:, None], a.sin()[:, None]
    z = y.clone()
    lo = torch.arange(r) * 2 if interleaved else torch.arange(r)
    hi = lo + 1 if interleaved else lo + r
    z[..., lo], z[..., hi] = y[..., lo] * c - y[..., hi] * s, y[..., hi] * c + y[..., lo] * s
    both = 8 * U32 * (y[..., lo].abs() + y[..., hi].abs()) + tol[..., lo] + tol[..., hi]
    tol[..., lo] = both
    tol[..., hi] = both
    return z, tol


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,n,Hq,Hkv,D,rot,page,norm,wide,axes", [
    (1, 1, 1, 1, 8, 0, 1, "all", False, 0), (2, 5, 4, 4, 64, 64, 16, "head", True, 3), (3, 17, 6, 2, 80, 48, 8, "all", True, 1), (2, 9, 8, 1, 256, 256, 32, "head", False, 2),
    (2, 33, 4, 4, 128, 64, 64, "none", False, 3), (1, 3, 9, 3, 96, 96, 2, "bare", False, 0), (2, 4, 2, 2, 24, 16, 4, "head", False, 4), (1, 2, 40, 8, 128, 128, 16, "all", False, 0)])
def test_append(beam, dtype, interleaved, B, n, Hq, Hkv, D, rot, page, norm, wide, axes):  # noqa: F811
    g = gen(n * D + axes)
    cap = 3 * page + n
    k_pages, v_pages, table = a_cache(5, B, cap, Hkv, D, page, dtype, "hnd" if n % 2 else "nhd", fill=7.0)
    k, v, q = (torch.randn(B, n, h, D, generator=g).mul(3).to(dtype) for h in (Hkv, Hkv, Hq))
    k[0, 0, 0] = 0                                                      # a head of zeros stays one
    first = torch.randint(0, 3 * page, (B,), generator=g).int()
    inv = (10000.0 ** (-torch.arange(0, rot, 2).double() / max(rot, 1))).float()
    eps = None if norm == "none" else 1e-5
    kind = torch.float32 if wide else dtype
    qw, kw = [None, None] if norm in ("none", "bare") else [(torch.rand((D,) if norm == "all" else (h, D), generator=g) + 0.5).to(kind) for h in (Hq, Hkv)]
    axis = torch.randint(-1, axes + 1, (rot // 2,), generator=g).int() if axes else None
    for position, count in ((None, None), (torch.randint(-5, 2**20, (B, n, max(axes, 1)), generator=g).int(), torch.randint(0, n + 2, (B,), generator=g).int())):
        if position is None and axes:
            continue
        kp, vp = k_pages.clone(), v_pages.clone()
        q_dev = q.cuda()
        pos_dev = None if position is None else position.cuda() if axes else position[:, :, 0].contiguous().cuda()
        args = cuda(k, v) + [kp, vp] + cuda(table, first, count)
        more = dict(position=pos_dev, inv_freq=inv.cuda() if rot else None, interleaved=interleaved, axis=None if axis is None else axis.cuda(), eps=eps,
                    q_weight=None if qw is None else qw.cuda(), k_weight=None if kw is None else kw.cuda())
        q_out = beam.append(*args, q=q_dev, **more)
        beam.append(*args, q=q_dev, q_out=q_dev, **more)
        assert torch.equal(q_dev, q_out)                                 # in place, too
        kc, vc = kp.cpu().double(), vp.cpu().double()
        touched = torch.zeros(kc.shape[:2], dtype=torch.bool)
        for b in range(B):
            m = n if count is None else min(n, int(count[b]))
            pos = first[b] + torch.arange(n) if position is None else position[b] if axes else position[b, :, 0]
            want_k, tol_k = normed_rotated(k[b], kw, eps, pos, axis, inv, interleaved)
            want_q, tol_q = normed_rotated(q[b], qw, eps, pos, axis, inv, interleaved)
            for i in range(m):
                t = int(first[b]) + i
                at = table[b, t // page], t % page
                touched[at] = True
                assert ((kc[at] - want_k[i]).abs() <= U[dtype] * want_k[i].abs() + tol_k[i] * (1 + U[dtype]) + LEAST[dtype]).all()
                assert torch.equal(vc[at], v[b, i].double())
            got = q_out[b].cpu().double()
            assert ((got[:m] - want_q[:m]).abs() <= U[dtype] * want_q[:m].abs() + tol_q[:m] * (1 + U[dtype]) + LEAST[dtype]).all()
            assert (got[m:] == 0).all()
        assert (kc[~touched] == 7).all() and (vc[~touched] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,n,Hq,Hkv,D,rot,norm,axes", [(4, 1027, 6, 2, 64, 32, "head", 3), (3, 1366, 3, 3, 80, 80, "all", 0), (70, 60, 9, 1, 16, 16, "none", 2)])
def test_append_of_many_tokens(beam, dtype, interleaved, B, n, Hq, Hkv, D, rot, norm, axes):  # noqa: F811
    """Several tokens a workgroup; counts that end inside one, and those of no token."""
    g, page = gen(n), 32
    k_pages, v_pages, table = a_cache(5, B, n + 40, Hkv, D, page, dtype, fill=7.0)
    k, v, q = (torch.randn(B, n, h, D, generator=g).to(dtype) for h in (Hkv, Hkv, Hq))
    first, count = torch.randint(0, 40, (B,), generator=g).int(), torch.randint(1, n + 1, (B,), generator=g).int()
    count[0], count[1], count[2] = -2**31, n, 3
    inv = (10000.0 ** (-torch.arange(0, rot, 2).double() / rot)).float()
    eps = None if norm == "none" else 1e-5
    qw, kw = [None, None] if norm == "none" else [(torch.rand((D,) if norm == "all" else (h, D), generator=g) + 0.5).to(dtype) for h in (Hq, Hkv)]
    axis = torch.randint(0, axes, (rot // 2,), generator=g).int() if axes else None
    position = torch.randint(0, 50000, (B, n, axes), generator=g).int() if axes else None
    q_dev = q.cuda()
    more = dict(position=None if position is None else position.cuda(), inv_freq=inv.cuda(), interleaved=interleaved, axis=None if axis is None else axis.cuda(), eps=eps,
                q_weight=None if qw is None else qw.cuda(), k_weight=None if kw is None else kw.cuda())
    beam.append(*cuda(k, v), k_pages, v_pages, *cuda(table, first, count), q=q_dev, q_out=q_dev, **more)
    kc, vc, touched = k_pages.cpu().double(), v_pages.cpu().double(), torch.zeros(k_pages.shape[:2], dtype=torch.bool)
    for b in range(B):
        m = max(0, int(count[b]))
        pos = position[b] if axes else first[b] + torch.arange(n)
        want_k, tol_k = normed_rotated(k[b], kw, eps, pos, axis, inv, interleaved)
        want_q, tol_q = normed_rotated(q[b], qw, eps, pos, axis, inv, interleaved)
        t = int(first[b]) + torch.arange(m)
        at = table[b, t // page].long(), t % page
        touched[at] = True
        assert ((kc[at] - want_k[:m]).abs() <= U[dtype] * want_k[:m].abs() + tol_k[:m] * (1 + U[dtype]) + LEAST[dtype]).all()
        assert torch.equal(vc[at], v[b, :m].double())
        got = q_dev[b].cpu().double()
        assert ((got[:m] - want_q[:m]).abs() <= U[dtype] * want_q[:m].abs() + tol_q[:m] * (1 + U[dtype]) + LEAST[dtype]).all()
        assert (got[m:] == 0).all()
    assert (kc[~touched] == 7).all() and (vc[~touched] == 7).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_append_norms_of_any_size(beam, dtype):  # noqa: F811
    """Squares pass fp32's range at both ends; what is not finite stays with its head."""
    sizes = torch.tensor([1e38, 3e30, 1e20, 1.0, 1e-15, 1e-22, 1e-30])
    B, n, H, D = 1, len(sizes), 3, 64
    k_pages, v_pages, table = a_cache(1, B, 16, H, D, 16, dtype)
    x = ((torch.rand(B, n, H, D, generator=gen(1)) + 0.5) * sizes[None, :, None, None]).to(dtype)
    x[0, 3, 1, 5] = NAN
    x[0, 3, 2, 7] = INF
    for eps in (1e-6, 1e-37):
        q = beam.append(*cuda(x, x), k_pages, v_pages, *cuda(table, ints(0)), q=x.cuda(), eps=eps).cpu().double()[0]
        want, tol = normed_rotated(x[0], None, float(np.float32(eps)), torch.zeros(n), None, torch.zeros(0), False)
        for i in range(n):
            for h in range(H):
                if i == 3 and h == 1:
                    assert torch.isnan(q[i, h]).all()
                elif i == 3 and h == 2:
                    assert torch.isnan(q[i, h, 7]) and (q[i, h, :7] == 0).all() and (q[i, h, 8:] == 0).all()
                else:
                    tiny = 2.0 ** -126 if dtype == torch.float32 else 2.0 ** -133
                    assert ((q[i, h] - want[i, h]).abs() <= U[dtype] * want[i, h].abs() + tol[i, h] * (1 + U[dtype]) + tiny).all(), (eps, i, h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("wide", [False, True])
def test_append_of_keys_alone_and_weights_of_one_side(beam, dtype, wide):  # noqa: F811
    B, n, H, D = 2, 5, 3, 64
    k_pages, v_pages, table = a_cache(1, B, 32, H, D, 8, dtype)
    qkv = torch.randn(B, n, 3 * H, D, generator=gen(1)).to(dtype)
    q, k, v = qkv.chunk(3, dim=2)
    dev, first = qkv.cuda().chunk(3, dim=2), ints(0, 9)
    w = (torch.rand(H, D, generator=gen(2)) + 0.5).to(torch.float32 if wide else dtype)
    none, inv = torch.zeros(n), torch.zeros(0)
    for weights in ((None, None), (w, None), (None, w)):
        for with_q in (True, False):
            more = dict(eps=1e-6, q_weight=None if weights[0] is None or not with_q else w.cuda(), k_weight=None if weights[1] is None else w.cuda())
            got = beam.append(dev[1], dev[2], k_pages, v_pages, *cuda(table, first), q=dev[0] if with_q else None, **more)
            assert (got is None) == (not with_q)
            for b in range(B):
                t = int(first[b]) + torch.arange(n)
                at = table[b, t // 8].long().cuda(), (t % 8).cuda()
                for have, x, weight in ((k_pages[at], k, weights[1]),) + (((got[b], q, weights[0]),) if with_q else ()):
                    want, tol = normed_rotated(x[b], weight, 1e-6, none, None, inv, False)
                    assert ((have.cpu().double() - want).abs() <= U[dtype] * want.abs() + tol * (1 + U[dtype]) + LEAST[dtype]).all()
                assert torch.equal(v_pages[at].cpu(), v[b])


@pytest.mark.parametrize("dtype", TYPES)
def test_append_without_norms_or_axes_to_speak_of_is_append(beam, dtype):  # noqa: F811
    """Each is 4 u32 (|x0| + |x1|) and a rounding from the definition at most (as in test_gpu_beam_ops.py; the angles are the same)."""
    k_pages, v_pages, table = a_cache(1, 2, 64, 2, 64, 8, dtype)
    qkv = torch.randn(2, 6, 8, 64, generator=gen(4)).to(dtype).cuda()
    inv, position = torch.rand(32, generator=gen(5)).cuda(), torch.randint(0, 90000, (2, 6), generator=gen(6)).int().cuda()
    ref = [k_pages.clone(), v_pages.clone()]
    more = dict(inv_freq=inv, q=qkv[:, :, :4])
    first = ints(0, 9).cuda()
    a = beam.append(qkv[:, :, 4:6], qkv[:, :, 6:], *ref, table.cuda(), first, position=position, **more)
    b = beam.append(qkv[:, :, 4:6], qkv[:, :, 6:], k_pages, v_pages, table.cuda(), first, position=position[:, :, None].contiguous(),
                    axis=torch.zeros(32, dtype=torch.int32).cuda(), **more)
    for x, y in ((a, b), (ref[0], k_pages)):
        x, y = x.double(), y.double()
        assert ((x - y).abs() <= 2 * U[dtype] * x.abs() + 8 * U32 * (x.abs() + x.roll(32, dims=-1).abs()) * 2 ** 0.5 + 2 * LEAST[dtype]).all()
    assert torch.equal(ref[1], v_pages)


# ---- attention behind a common prefix --------------------------------------------------------------------------------
def tokens_of(table, n_pages, page, L):
    t = np.arange(min(L, len(table) * page))
    p = table.numpy().astype(np.int64)[t // page]
    ok = (p >= 0) & (p < n_pages)
    return t, torch.from_numpy(np.where(ok, p * page + t % page, 0)), torch.from_numpy(ok)


def plain_shared(q, k_pages, v_pages, shared, P0, table, prefix, tree, seen_of_tree, scale):
    """seen_of_tree(b) -> [n, tree[b]] bool."""
    B, n, Hq, D = q.shape
    page, Hkv, N = k_pages.shape[1], k_pages.shape[2], len(k_pages)
    out, tol = torch.zeros(B, n, Hq, D, dtype=torch.float64), torch.zeros(B, n, Hq, D, dtype=torch.float64)
    lse, lse_tol = torch.full((B, n, Hq), -INF, dtype=torch.float64), torch.zeros(B, n, Hq, dtype=torch.float64)
    kp, vp, u = k_pages.cpu().double().reshape(-1, Hkv, D), v_pages.cpu().double().reshape(-1, Hkv, D), U[q.dtype]
    _, at0, ok0 = tokens_of(shared, N, page, max(0, P0))
    for b in range(B):
        P, T = max(0, int(prefix[b])), max(0, int(tree[b]))
        t, at, ok = tokens_of(table[b], N, page, P + T)
        see = torch.ones(n, len(t), dtype=torch.bool)
        see[:, P:] = seen_of_tree(b)[:, :len(t) - P] if T and len(t) > P else False
        see = torch.cat((ok0.expand(n, -1), see & ok), dim=1)
        at = torch.cat((at0, at))
        if not len(at):
            continue
        for h in range(Hq):
            k, v, x = kp[at, h * Hkv // Hq], vp[at, h * Hkv // Hq], q[b, :, h].cpu().double()
            s = (x @ k.T * scale).masked_fill(~see, -INF)
            lse[b, :, h] = torch.logsumexp(s, dim=1)
            alive = lse[b, :, h] > -INF
            p = torch.where(see & alive[:, None], (s - lse[b, :, h, None]).exp(), 0.0)
            v = torch.where(see.any(dim=0)[:, None], v, 0.0)
            out[b, :, h] = p @ v
            e = (D + 8) * U32 * (x.abs() @ k.abs().T).masked_fill(~see, 0.0).amax(dim=1) * abs(scale)
            m = see.sum(dim=1)
            tol[b, :, h] = u * out[b, :, h].abs() + (p @ v.abs()) * (u + 2 * (2 * e + 2.0 ** -21) + m * U32)[:, None]
            lse_tol[b, :, h] = 2 * e + 2.0 ** -20 + m * U32 + U32 * torch.where(alive, lse[b, :, h].abs(), 0.0)
    return out, lse, tol, lse_tol


def setting(dtype, B, Hkv, D, page, common, prefix, tree, seed=0, layout="nhd"):
    """Pools with a table of the sentences and one of what they have in common."""
    cap = max(1, max(max(0, p) + max(0, t) for p, t in zip(prefix, tree)))
    per, more = -(-cap // page), max(1, -(-common // page))
    k_pages, v_pages, table = a_cache(seed, B + -(-more // per), cap, Hkv, D, page, dtype, layout)
    return k_pages, v_pages, table[B:].reshape(-1)[:more].contiguous(), table[:B].contiguous()


def check_shared(beam, dtype, B, n, Hq, Hkv, D, page, common, prefix, tree, masked, layout="nhd", seed=0, scale=None, spoil=None, **more):  # noqa: F811
    k_pages, v_pages, shared, table = setting(dtype, B, Hkv, D, page, common, prefix, tree, seed, layout)
    prefix, tree = ints(*prefix), ints(*tree)
    q = torch.randn(B, n, Hq, D, generator=gen(seed + 1)).to(dtype).cuda()
    mask = None
    if masked:
        mask, bits = random_mask(seed, B, n, -(-max(1, int(tree.max())) // 64))
        seen = lambda b: torch.from_numpy(bits[b, :, :max(0, int(tree[b]))])
    else:
        seen = lambda b: torch.arange(max(0, int(tree[b])))[None] <= int(tree[b]) - n + torch.arange(n)[:, None]
    if spoil:
        spoil(k_pages, v_pages, shared, table)
    got, lse = beam.attend_shared(q, k_pages, v_pages, *cuda(shared, ints(common), table, prefix, tree, mask), scale=scale, return_lse=True, **more)
    near(got, lse, plain_shared(q, k_pages, v_pages, shared, common, table, prefix, tree, seen, D ** -0.5 if scale is None else scale))


SHAPES = [
    # B, n, Hq, Hkv, D, page, common, prefix, tree
    (1, 1, 1, 1, 8, 1, 1, [1], [0]),
    (2, 1, 8, 8, 64, 16, 1000, [20, 3], [1, 1]),
    (3, 5, 4, 4, 64, 16, 63, [0, 17, 130], [70, 64, 5]),
    (4, 20, 8, 2, 128, 16, 333, [63, 65, 1, 0], [100, 40, 20, 20]),
    (2, 7, 6, 2, 80, 8, 129, [200, 3], [33, 130]),
    (5, 3, 16, 1, 96, 32, 65, [31, 50, 0, 1, 2], [1, 63, 3, 3, 4]),
    (1, 33, 8, 8, 32, 64, 200, [77], [129]),
    (2, 2, 6, 3, 256, 4, 70, [100, 5], [65, 20]),
    (9, 11, 16, 2, 128, 16, 517, [30] * 9, [11] * 9),
    (3, 70, 4, 2, 256, 16, 90, [30, 2, 0], [70] * 3),
    (4, 1, 3, 1, 24, 2, 5, [0, 1, 2, 3], [1, 0, 2, 1]),
    (9, 10, 8, 1, 40, 16, 205, [3] * 9, [10] * 9),
    (40, 5, 3, 3, 64, 64, 77, [1] * 40, [5] * 40),
    (17, 2, 8, 2, 96, 128, 640, [0] * 17, [2] * 17),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_shared(beam, dtype, masked, shape):  # noqa: F811
    check_shared(beam, dtype, *shape, masked=masked, layout="nhd" if masked else "hnd", seed=shape[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("common", [0, -3, 1, 31, 32, 33, 64, 127, 128, 129, 700])
def test_shared_lengths_of_what_is_in_common(beam, dtype, common):  # noqa: F811
    check_shared(beam, dtype, 3, 9, 8, 2, 64, 16, common, [0, 5, 0], [0, 9, 3], masked=True, seed=2)
    check_shared(beam, dtype, 7, 6, 8, 2, 128, 16, common, [0, 5, 0, 1, 2, 3, 4], [0, 9, 3, 1, 1, 1, 6], masked=False, seed=3)


@pytest.mark.parametrize("dtype", TYPES)
def test_shared_over_many_tokens(beam, dtype):  # noqa: F811
    check_shared(beam, dtype, 2, 3, 4, 2, 64, 64, 9000, [50, 3], [50, 3], masked=True)
    check_shared(beam, dtype, 6, 20, 8, 2, 128, 16, 3001, [17] * 6, [20] * 6, masked=False)
    check_shared(beam, dtype, 2, 2, 4, 2, 128, 16, 40, [3001, 10], [2, 2], masked=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [3.0, -0.5, 0.0])
def test_shared_scales(beam, dtype, scale):  # noqa: F811
    check_shared(beam, dtype, 2, 5, 4, 2, 64, 16, 100, [300, 20], [40, 64], masked=True, scale=scale)
    check_shared(beam, dtype, 30, 5, 4, 2, 128, 16, 150, [3] * 30, [5] * 30, masked=False, scale=scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,n,D", [(2, 4, 64), (20, 8, 128)])
def test_shared_pages_that_are_not_there(beam, dtype, B, n, D):  # noqa: F811
    def spoil(k_pages, v_pages, shared, table):
        shared[1], shared[-1], table[0, 0] = -1, 2**31 - 1, -2**31
    check_shared(beam, dtype, B, n, 4, 2, D, 8, 100, [30] * B, [n] * B, masked=False, spoil=spoil)
    def nothing(k_pages, v_pages, shared, table):
        shared[:] = -1
        table[0] = -5
    k_pages, v_pages, shared, table = setting(dtype, B, 2, D, 8, 100, [30] * B, [n] * B)
    nothing(k_pages, v_pages, shared, table)
    q = torch.randn(B, n, 4, D, generator=gen(1)).to(dtype).cuda()
    out, lse = beam.attend_shared(q, k_pages, v_pages, *cuda(shared, ints(100), table, ints(*[30] * B)), return_lse=True)
    assert (out[0] == 0).all() and (lse[0] == -INF).all() and torch.isfinite(lse[1:]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,n", [(2, 4), (20, 10)])
def test_shared_values_that_are_not_finite(beam, dtype, B, n):  # noqa: F811
    """In places that nobody sees they do not matter; an element of a common token that is not finite reaches that element of all."""
    H, D, page, common = 2, 64, 8, 85
    k_pages, v_pages, shared, table = setting(dtype, B, H, D, page, common, [40] * B, [n] * B)      # (more room than is used)
    q = torch.randn(B, n, 2 * H, D, generator=gen(1)).to(dtype).cuda()
    args = cuda(shared, ints(common), table, ints(*[20] * B), ints(*[n] * B))
    want = beam.attend_shared(q, k_pages, v_pages, *args, return_lse=True)
    last = int(shared[-1])
    for x in (k_pages, v_pages):
        x[last, common % page:] = NAN
        for b in range(B):
            x[int(table[b, (20 + n) // page]), (20 + n) % page:] = INF
    got = beam.attend_shared(q, k_pages, v_pages, *args, return_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    v_pages[int(shared[2]), 3, 1, 7] = NAN
    got = beam.attend_shared(q, k_pages, v_pages, *args)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[:, :, 2:, 7] = True
    assert torch.equal(torch.isnan(got), hit) and torch.equal(got[~hit], want[0][~hit])


@pytest.mark.parametrize("dtype", TYPES)
def test_shared_strides_and_results_in_place(beam, dtype):  # noqa: F811
    B, n, H, D = 12, 6, 2, 128
    k_pages, v_pages, shared, table = setting(dtype, B, H, D, 16, 200, [40] * B, [n] * B)
    room = torch.randn(n, B, 2 * H + 2, D, generator=gen(1)).to(dtype).cuda()
    q = room.transpose(0, 1)[:, :, 1:-1]                                # sentences closer together than tokens
    args = cuda(shared, ints(200), table, ints(*[40] * B), ints(*[n] * B))
    want, lse = beam.attend_shared(q.contiguous(), k_pages, v_pages, *args, return_lse=True)
    kept = room.clone()
    got, lse2 = beam.attend_shared(q, k_pages, v_pages, *args, out=q, return_lse=True)
    assert torch.equal(got, want) and torch.equal(lse, lse2)
    assert torch.equal(room[:, :, 0], kept[:, :, 0]) and torch.equal(room[:, :, -1], kept[:, :, -1])


@pytest.mark.parametrize("dtype", TYPES)
def test_shared_is_attention_over_both(beam, dtype):  # noqa: F811
    """A batch of one: the same as attention over a table of both, as near as either is to the definition."""
    H, D, page = 2, 64, 16
    k_pages, v_pages, shared, table = setting(dtype, 1, H, D, page, 160, [30], [5])
    q = torch.randn(1, 5, 2 * H, D, generator=gen(1)).to(dtype).cuda()
    both = torch.cat((shared[None], table), dim=1).contiguous()
    a, la = beam.attend_shared(q, k_pages, v_pages, *cuda(shared, ints(160), table, ints(30), ints(5)), return_lse=True)
    b, lb = beam.attend(q, k_pages, v_pages, *cuda(both, ints(190), ints(5)), return_lse=True)
    v = float(v_pages.abs().max())
    assert (a.double() - b.double()).abs().max() <= 6 * U[dtype] * v and (la - lb).abs().max() < 1e-4


# ---- weighing --------------------------------------------------------------------------------------------------------
def check_weigh(beam, dtype, B, n, Hq, Hkv, D, page, prefix, tree, masked, by_head, layout="nhd", seed=0, scale=None, count=None, max_len=None, spoil=None):  # noqa: F811
    prefix, tree = ints(*prefix), ints(*tree)
    cap = max(1, int((prefix.clamp(min=0) + tree.clamp(min=0)).max()))
    k_pages, v_pages, table = a_cache(seed, B, cap, Hkv, D, page, dtype, layout)
    q = torch.randn(B, n, Hq, D, generator=gen(seed + 1)).to(dtype)
    mask = None
    if masked:
        mask, bits = random_mask(seed, B, n, -(-max(1, int(tree.max())) // 64))
        seen = lambda b, T: torch.from_numpy(bits[b, :, :T])
    else:
        seen = lambda b, T: torch.arange(T)[None] <= int(tree[b]) - n + torch.arange(n)[:, None]
    if spoil:
        spoil(k_pages, table)
    width = table.shape[1] * page + 5
    H = Hkv if by_head else 1
    score = torch.rand(B, H, width, generator=gen(seed + 2)) * 2
    lse = torch.randn(B, n, Hq, generator=gen(seed + 3)) + 3
    lse[0, n // 2, 0] = INF
    lse[-1, 0, -1] = -INF
    lse[-1, -1, 0] = NAN
    sc, G = D ** -0.5 if scale is None else scale, Hq // Hkv
    kp = k_pages.cpu().double().reshape(-1, Hkv, D)
    want, tol = score.double(), score.double() * U32
    for b in range(B):
        P, T = max(0, int(prefix[b])), max(0, int(tree[b]))
        limit = P + T if max_len is None else min(max_len, P + T)
        t, at, ok = tokens_of(table[b], len(k_pages), page, limit)
        see = torch.ones(n, len(t), dtype=torch.bool)
        if len(t) > P:
            see[:, P:] = seen(b, T)[:, :len(t) - P]
        see &= ok
        if count is not None:
            see[max(0, count[b]):] = False
        for h in range(Hq):
            l = lse[b, :, h].double()
            live = see & torch.isfinite(l)[:, None]
            x = q[b, :, h].double() @ kp[at, h // G].T * sc
            w = torch.where(live, (x - l[:, None]).exp(), 0.0)
            e = (D + 8) * U32 * (q[b, :, h].double().abs() @ kp[at, h // G].abs().T) * abs(sc) + 4 * U32 * (x.abs() + l.abs()[:, None])
            want[b, h // G if by_head else 0, :len(t)] += w.sum(dim=0)
            tol[b, h // G if by_head else 0, :len(t)] += torch.where(live, w * (2 * e + 2.0 ** -21 + n * Hq * U32), 0.0).sum(dim=0)
    tol += U32 * want
    args = [q.cuda(), lse.cuda(), k_pages] + cuda(table, prefix, tree, mask)
    more = dict(scale=scale, max_len=max_len, count=None if count is None else ints(*count).cuda())
    dev = score.cuda()
    out = beam.weigh(dev, *args, out=torch.full_like(dev, 9.0), **more)
    assert torch.equal(dev.cpu(), score)
    assert ((out.cpu().double() - want).abs() <= tol).all(), float(((out.cpu().double() - want).abs() - tol).max())
    again = beam.weigh(dev, *args, **more)                              # in place: the same, bit for bit
    assert again.data_ptr() == dev.data_ptr() and torch.equal(dev, out)


WEIGH = [
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
    (2, 150, 4, 2, 64, 16, [0, 37], [150, 150]),
    (2, 25, 8, 2, 128, 16, [300, 0], [100, 25]),
    (1, 32, 8, 2, 64, 32, [1500], [32]),
    (3, 40, 9, 3, 40, 8, [70, 0, 200], [64, 128, 40]),
    (1, 300, 8, 2, 64, 16, [100], [300]),
    (2, 200, 6, 1, 256, 16, [0, 5], [200, 7]),
    (2, 90, 3, 1, 256, 16, [0, 300], [90, 200]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("by_head", [True, False])
@pytest.mark.parametrize("shape", WEIGH)
def test_weigh(beam, dtype, masked, by_head, shape):  # noqa: F811
    check_weigh(beam, dtype, *shape, masked=masked, by_head=by_head, layout="nhd" if masked else "hnd", seed=shape[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_weigh_counts_scales_and_ends(beam, dtype):  # noqa: F811
    shape = 4, 9, 8, 2, 64, 16, [100, 0, -4, 33], [9, 50, 20, -1]
    for by_head in (True, False):
        check_weigh(beam, dtype, *shape, masked=False, by_head=by_head, count=[9, 3, -1, 70])
        check_weigh(beam, dtype, *shape, masked=True, by_head=by_head, count=[0, 1, 8, 9], scale=-0.2)
        check_weigh(beam, dtype, *shape, masked=True, by_head=by_head, scale=0.0)
        for max_len in (1, 64, 101, 105):
            check_weigh(beam, dtype, *shape, masked=True, by_head=by_head, max_len=max_len)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 80])
def test_weigh_what_is_not_seen_does_not_matter(beam, dtype, n):  # noqa: F811
    def spoil(k_pages, table):
        table[0, 3] = -1
        for b in range(2):
            p = int(table[b, -1])
            k_pages[p, -3:] = NAN                                        # behind the end
    check_weigh(beam, dtype, 2, n, 4, 2, 64, 8, [30, 20], [75, 85], masked=True, by_head=True, spoil=spoil)
    # (neither sentence's last page is full: 105 tokens in pages of 8)
    k_pages, v_pages, table = a_cache(1, 1, 40, 1, 64, 8, dtype)
    q, lse = torch.randn(1, 2, 1, 64).to(dtype).cuda(), torch.zeros(1, 2, 1).cuda()
    mask = torch.tensor([[[0b0111], [0b1011]]]).cuda()
    args = q, lse, k_pages, *cuda(table, ints(30), ints(4), mask)
    want = beam.weigh(torch.zeros(1, 1, 40).cuda(), *args)
    k_pages[int(table[0, 4]), 0] = INF                                  # token 32 of the tree's: only the first node sees it
    got = beam.weigh(torch.zeros(1, 1, 40).cuda(), *args)
    assert torch.equal(got[..., :32], want[..., :32]) and torch.equal(got[..., 33:], want[..., 33:])
    lse[0, 0] = -INF                                                    # and that one does not count
    got = beam.weigh(torch.zeros(1, 1, 40).cuda(), *args)
    assert got[0, 0, 32] == 0 and torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_weights_of_attention_add_up_to_one(beam, dtype):  # noqa: F811
    B, n, Hq, Hkv, D = 3, 12, 8, 2, 64
    k_pages, v_pages, table = a_cache(1, B, 300, Hkv, D, 16, dtype)
    q = torch.randn(B, n, Hq, D, generator=gen(1)).to(dtype).cuda()
    mask, bits = random_mask(1, B, n, 2)
    args = cuda(table, ints(150, 20, 1), ints(100, 80, 30), mask)
    out, lse = beam.attend(q, k_pages, v_pages, *args, return_lse=True)
    for H in (Hkv, 1):
        score = beam.weigh(torch.zeros(B, H, 304).cuda(), q, lse, k_pages, *args)
        assert (score.double().sum(dim=2) - n * Hq / H).abs().max() < n * Hq * 1e-4


# ---- eviction --------------------------------------------------------------------------------------------------------
def plain_evict(score, k_pages, v_pages, table, new_table, prefix, tree, keep, budget, sinks, recent, max_len):
    B, H, width = score.shape
    page, Hkv, N = k_pages.shape[1], k_pages.shape[2], len(k_pages)
    k2, v2, new_score, new_prefix = k_pages.clone(), v_pages.clone(), torch.zeros_like(score), []
    there = lambda tab, t: t // page < len(tab) and 0 <= tab[t // page] < N
    for b in range(B):
        P = min(max(0, prefix[b]), max_len)
        T = min(P + max(0, tree[b]), max_len) - P if tree is not None else 0
        old, new = table[b].tolist(), new_table[b].tolist()
        ok = [t for t in range(P) if there(old, t)]
        stay = min(keep if budget is None else min(keep, max(0, budget[b])), len(ok))
        new_prefix.append(stay)
        for h in range(H):
            s = score[b, h].tolist()
            rank = lambda t: (not (t < sinks or t >= P - recent), s[t] != s[t], -s[t] if s[t] == s[t] else 0, t)
            kept = sorted(sorted(ok, key=rank)[:stay]) + list(range(P, P + T))
            heads = range(Hkv) if H == 1 else [h]
            for j, t in enumerate(kept):
                new_score[b, h, j] = score[b, h, t]
                if there(old, t) and there(new, j):
                    for x, y in ((k2, k_pages), (v2, v_pages)):
                        x[new[j // page], j % page, heads] = y[old[t // page], t % page, heads]
    return new_prefix, new_score, k2, v2


def check_evict(beam, dtype, B, Hkv, D, page, prefix, tree, by_head, keep, sinks=0, recent=0, budget=None, max_len=None, score=None, spoil=None, seed=0, new_pages=None, layout="nhd"):  # noqa: F811
    cap = max(1, max(max(0, p) + max(0, t) for p, t in zip(prefix, tree or [0] * B)))
    per = -(-cap // page)
    new_per = per if new_pages is None else new_pages
    k_pages, v_pages, both = a_cache(seed, 2 * B, cap, Hkv, D, page, dtype, layout)
    table, new_table = both[:B].contiguous(), both[B:, :new_per].contiguous()
    k_pages.copy_(torch.arange(k_pages.numel(), device="cuda").reshape(k_pages.shape) % 2039)
    v_pages.copy_(torch.arange(k_pages.numel(), device="cuda").reshape(k_pages.shape) % 1021)
    if spoil:
        spoil(table, new_table)
    if score is None:
        score = torch.randn(B, Hkv if by_head else 1, per * page + 3, generator=gen(seed)).exp()
    limit = min(per * page, score.shape[2]) if max_len is None else max_len
    want = plain_evict(score, k_pages.cpu(), v_pages.cpu(), table, new_table, prefix, tree, keep, budget, sinks, recent, limit)
    got = beam.evict(score.cuda(), k_pages, v_pages, *cuda(table, new_table, ints(*prefix), None if tree is None else ints(*tree)), keep=keep, sinks=sinks, recent=recent,
                     max_len=max_len, budget=None if budget is None else ints(*budget).cuda())
    assert got[0].tolist() == want[0]
    assert torch.equal(torch.nan_to_num(got[1].cpu(), nan=-7.0), torch.nan_to_num(want[1], nan=-7.0))
    assert torch.equal(k_pages.cpu(), want[2]) and torch.equal(v_pages.cpu(), want[3])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("by_head", [True, False])
@pytest.mark.parametrize("B,Hkv,D,page,prefix,tree,keep,sinks,recent", [
    (1, 1, 8, 1, [1], [0], 1, 0, 0), (2, 2, 64, 16, [100, 37], [5, 0], 20, 4, 8), (3, 4, 80, 8, [0, 1, 90], [20, 3, 0], 33, 1, 0), (1, 3, 24, 4, [500], [7], 499, 0, 100),
    (2, 2, 128, 32, [1100, 64], [0, 70], 64, 4, 30), (2, 1, 256, 2, [50, 49], [0, 0], 10, 6, 7), (1, 2, 32, 64, [3000], [1], 1500, 4, 600), (2, 2, 40, 16, [60, 20], [2, 3], 1000, 0, 0)])
def test_evict(beam, dtype, by_head, B, Hkv, D, page, prefix, tree, keep, sinks, recent):  # noqa: F811
    check_evict(beam, dtype, B, Hkv, D, page, prefix, tree, by_head, keep, sinks, recent, layout="nhd" if by_head else "hnd", seed=D)
    check_evict(beam, dtype, B, Hkv, D, page, prefix, None, by_head, keep, sinks, recent, seed=D + 1)


@pytest.mark.parametrize("by_head", [True, False])
def test_evict_more_first_and_last_ones_than_stay(beam, by_head):  # noqa: F811
    for sinks, recent in ((10, 10), (100, 0), (0, 100), (2**31 - 1, 2**31 - 1), (30, 31)):
        check_evict(beam, torch.bfloat16, 3, 2, 16, 8, [60, 15, 100], [3, 0, 9], by_head, 12, sinks, recent)


@pytest.mark.parametrize("by_head", [True, False])
def test_evict_budgets_and_ends(beam, by_head):  # noqa: F811
    shape = torch.float16, 4, 2, 16, 8, [60, 15, 100, -3], [3, 0, 9, 5], by_head
    check_evict(beam, *shape, 50, 2, 5, budget=[0, -5, 30, 9])
    check_evict(beam, *shape, 50, 2, 5, budget=[100, 3, 51, 1], new_pages=4)
    for max_len in (1, 8, 61, 101):
        check_evict(beam, *shape, 20, 2, 5, max_len=max_len)


@pytest.mark.parametrize("P", [900, 5000, 20000])
def test_evict_scores_of_all_kinds(beam, P):  # noqa: F811
    g = gen(P)
    few = torch.randint(0, 3, (P + 8,), generator=g).float()
    tiny = torch.rand(P + 8, generator=g) * 1e-40
    odd = torch.randn(P + 8, generator=g)
    odd[torch.randperm(P, generator=g)[:P // 3]] = NAN
    odd[::5], odd[1::7], odd[2::11] = -INF, INF, -0.0
    rows = [torch.zeros(P + 8), few, tiny, odd, torch.full((P + 8,), NAN), -torch.rand(P + 8, generator=g), torch.where(few > 0, 0.0, -0.0),
            torch.linspace(1.0, 1.0 + 2.0 ** -12, P + 8)]
    score = torch.stack(rows)[None]
    for keep in (1, P // 3, P // 2 + 1, P - 1):
        check_evict(beam, torch.float16, 1, 8, 8, 64, [P], [3], True, keep, 3, 10, score=score)
    check_evict(beam, torch.float16, 1, 8, 8, 64, [P], [3], True, P // 2, 0, 0, score=score)


def test_evict_pages_that_are_not_there(beam):  # noqa: F811
    def spoil(table, new_table):
        table[0, 0], table[0, 3], table[1, :], table[2, 12] = -1, 2**31 - 1, -1, -2**31
        new_table[0, 1], new_table[2, 0] = -1, 2**31 - 1
    for by_head in (True, False):
        for keep in (5, 40, 70, 200):
            check_evict(beam, torch.bfloat16, 3, 2, 16, 8, [70, 30, 95], [9, 5, 11], by_head, keep, 4, 12, spoil=spoil)


@pytest.mark.parametrize("P", [4000, 18000])
def test_evict_scores_around_nothing(beam, P):  # noqa: F811
    """Zeros of either sign are equal, and lie between the smallest numbers; infinities are greater than the greatest."""
    g = gen(P)
    small = (torch.rand(P + 8, generator=g) - 0.5) * 1e-40
    small[::3], small[1::3] = 0.0, -0.0
    large = (torch.rand(P + 8, generator=g) - 0.5) * 6e38
    large[::4], large[1::4] = INF, -INF
    score = torch.stack([small, -small.abs(), large, -large.abs()])[None]
    for keep in (P // 5, P // 2, P - P // 6):
        check_evict(beam, torch.float16, 1, 4, 8, 64, [P], [0], True, keep, 0, 0, score=score)


def test_evict_long_rows_with_pages_that_are_not_there(beam):  # noqa: F811
    def spoil(table, new_table):
        table[0, 5:9], table[0, 100], table[1, ::2] = -1, 2**31 - 1, -1
    for by_head in (True, False):
        for keep, recent in ((3000, 40), (9000, 9000), (17999, 0)):
            check_evict(beam, torch.float16, 2, 2, 8, 64, [18000, 17000], [70, 5], by_head, keep, 400, recent, spoil=spoil)


@pytest.mark.parametrize("P,keep", [(66000, 30000), (140000, 5)])
def test_evict_of_long_sentences(beam, P, keep):  # noqa: F811
    score = torch.randn(1, 1, P + 64, generator=gen(1)).round(decimals=2)
    check_evict(beam, torch.float16, 1, 1, 8, 256, [P], [20], False, keep, 4, 3, score=score)


# ---- together --------------------------------------------------------------------------------------------------------
def test_offsets_beyond_32_bits(beam):  # noqa: F811
    """A pool of 5 GiB: the last pages lie behind 2^31 elements."""
    page, H, D = 1024, 8, 128
    n = (1 << 31) // (page * H * D) + 40
    k_pages = torch.empty((n, page, H, D), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    last = [n - 1, n - 7, 0, n - 9, n - 11]
    for p in last:
        k_pages[p].normal_(generator=g)
    small = torch.stack([k_pages[p] for p in last])
    q = torch.randn(3, 2, 8, D, generator=gen(1)).bfloat16().cuda()
    score = torch.rand(1, H, 3000, generator=gen(2)).cuda()
    results = []
    for pool, ids in ((k_pages, last), (small, range(5))):
        ids = ints(*ids)
        a = beam.attend_shared(q, pool, pool, *cuda(ids[:2], ints(1500), ids[2:].repeat(3, 1), ints(900, 30, 2)), return_lse=True)
        w = beam.weigh(score, q[:1], a[1][:1].contiguous(), pool, *cuda(ids[None, :3].contiguous(), ints(2900)), out=torch.zeros_like(score))
        s = beam.evict(score, pool, pool, *cuda(ids[None, :3].contiguous(), ids[None, 3:].contiguous(), ints(2900)), keep=2000)
        y = beam.append(q[:1], q[:1], pool, pool, *cuda(ids[None, 3:].contiguous(), ints(1023)), q=q[:1], eps=1e-6)
        results.append(list(a) + [w, s[0], s[1], y] + [pool[int(p)].clone() for p in ids])
    assert all(torch.equal(x, y) for x, y in zip(*results))


def steps_of_a_decode(beam, x, pools, shared, common, table, new_table, first, tree, mask, inv, score):  # noqa: F811
    q = beam.append(x["k"], x["v"], *pools, table, first, inv_freq=inv, q=x["q"], eps=1e-6)
    o, lse = beam.attend_shared(q, *pools, shared, common, table, first, tree, mask, return_lse=True)
    weights = beam.weigh(score, q, lse, pools[0], table, first, tree, mask, out=torch.empty_like(score))
    stay, moved = beam.evict(weights, *pools, table, new_table, first, tree, keep=40, sinks=2, recent=8)
    again = beam.attend_shared(q, *pools, shared, common, new_table, stay, tree, mask)
    return q, o, lse, weights, stay, moved, again


@pytest.mark.parametrize("graph", [False, True])
def test_a_step_on_a_stream_of_its_own_and_in_a_graph(beam, graph):  # noqa: F811
    B, k, H, D, page = 3, 6, 4, 64, 16
    g = gen(8)
    k_pages, v_pages, both = a_cache(8, 2 * B + 1, 200, 2, D, page, torch.bfloat16)
    pools = k_pages, v_pages
    shared, table, new_table = cuda(both[0].contiguous(), both[1:1 + B].contiguous(), both[1 + B:].contiguous())
    first, tree, common = cuda(ints(10, 100, 55), ints(k, k, k), ints(150))
    mask = (torch.ones(1, dtype=torch.int64) << torch.arange(k)).expand(B, k).reshape(B, k, 1).contiguous().cuda()
    x = {n: torch.zeros(B, k, h, D, dtype=torch.bfloat16, device="cuda") for n, h in (("q", H), ("k", 2), ("v", 2))}
    inv, score = torch.rand(32, generator=g).cuda(), torch.zeros(B, 2, 200).cuda()
    step = lambda: steps_of_a_decode(beam, x, pools, shared, common, table, new_table, first, tree, mask, inv, score)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    held = None
    if graph:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            held = step()
    for i in range(4):
        for t in x.values():
            t.copy_(torch.randn(t.shape, generator=g))
        score.copy_(torch.rand(score.shape, generator=g) * 0.01)
        torch.cuda.synchronize()
        if graph:
            captured.replay()
        else:
            with torch.cuda.stream(s):
                held = step()
            s.synchronize()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert want[4].tolist() == [10, 40, 40]
