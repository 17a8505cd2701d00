"""-m gpu: attention over a tree at the edges of what it accepts.  Tolerances are those of test_gpu_beam_ops.py."""
import math

import numpy as np
import pytest
import torch

from test_gpu_beam_ops import TYPES, U, U32, a_cache, beam, gen, near, plain_attend, random_mask, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu
MOST = 2**31 - 1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 5, 70])
def test_attend_along_a_chain_of_any_length(beam, dtype, n):  # noqa: F811
    """A tree of as much as there is, up to the greatest number: cut off by max_len, as a long prefix is."""
    B, H, D, page = 6, 2, 64, 8
    prefix = torch.tensor([0, 1, 100, 100, 7, MOST], dtype=torch.int32)
    tree = torch.tensor([MOST, MOST, MOST - 11, 60, MOST - 500, MOST], dtype=torch.int32)
    k_pages, v_pages, table = a_cache(2, B, 200, H, D, page, dtype)
    q = torch.randn(B, n, 2 * H, D, generator=gen(n)).to(dtype).cuda()
    seen = lambda b, i, j: j <= int(tree[b]) - n + i
    got, lse = beam.attend(q, k_pages, v_pages, table.cuda(), prefix.cuda(), tree.cuda(), return_lse=True)
    near(got, lse, plain_attend(q, k_pages, v_pages, table, prefix, tree, seen, D ** -0.5))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,n,Hq,Hkv,D,length", [(3, 4, 8, 2, 64, 900), (2, 90, 6, 3, 80, 300), (140, 2, 8, 8, 64, 40), (1, 1, 4, 1, 128, 5000)])
def test_attend_into_its_queries(beam, dtype, B, n, Hq, Hkv, D, length):  # noqa: F811
    k_pages, v_pages, table = a_cache(1, B, length, Hkv, D, 16, dtype)
    q = torch.randn(B, n, Hq + 2, D, generator=gen(2)).to(dtype).cuda()
    prefix = torch.full((B,), length, dtype=torch.int32)
    prefix[0] = length // 2
    args = k_pages, v_pages, table.cuda(), prefix.cuda()
    want, lse = beam.attend(q[:, :, 1:-1], *args, return_lse=True)
    kept = q.clone()
    got, lse2 = beam.attend(q[:, :, 1:-1], *args, out=q[:, :, 1:-1], return_lse=True)
    assert torch.equal(q[:, :, 1:-1], want) and torch.equal(lse, lse2) and got.data_ptr() == q[:, :, 1:-1].data_ptr()
    assert torch.equal(q[:, :, 0], kept[:, :, 0]) and torch.equal(q[:, :, -1], kept[:, :, -1])


INF, NAN = math.inf, math.nan


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,n,Hq,Hkv,D,prefix,tree,masked", [
    (2, 3, 2, 2, 64, 20, 90, True), (2, 1, 4, 4, 8, 0, 300, False), (2, 20, 4, 2, 64, 65, 200, True), (2, 50, 2, 2, 64, 3, 120, True), (1, 90, 4, 2, 64, 70, 250, False),
    (2, 8, 4, 2, 128, 5, 150, True), (1, 50, 2, 2, 128, 40, 130, True), (2, 70, 4, 1, 128, 30, 200, True), (1, 130, 3, 3, 80, 0, 130, False),
    (2, 5, 4, 2, 256, 33, 100, True), (1, 70, 4, 2, 256, 9, 140, False), (130, 2, 8, 8, 64, 3, 40, True), (1, 6, 1, 1, 96, 10, 3000, True)])
def test_attend_values_that_are_not_finite(beam, dtype, B, n, Hq, Hkv, D, prefix, tree, masked):  # noqa: F811
    """Elements of the tree's values, here and there, are infinities or NaN: an element of a node is what the sum of those it sees is, and
    as good as ever if it sees none."""
    page, rng = 8, np.random.RandomState(n + D)
    k_pages, v_pages, table = a_cache(3, B, prefix + tree, Hkv, D, page, dtype)
    q = torch.randn(B, n, Hq, D, generator=gen(4)).to(dtype).cuda()
    mask, bits = random_mask(5, B, n, -(-tree // 64), 0.3)
    sees = lambda b, i, j: bits[b, i, j] if masked else j <= tree - n + i
    p, t = (torch.full((B,), x, dtype=torch.int32) for x in (prefix, tree))
    clean = v_pages.clone()
    effect = np.zeros((2, B, n, Hkv, D), bool)                            # an infinity is seen; a negative one
    for b in range(B):
        for _ in range(12):
            j, h, d, x = rng.randint(tree), rng.randint(Hkv), rng.randint(D), (INF, -INF, NAN)[rng.randint(3)]
            at = int(table[b, (prefix + j) // page]), (prefix + j) % page, h, d
            if not torch.isfinite(v_pages[at]):
                continue
            clean[at], v_pages[at] = 0, x
            for i in range(n):
                if sees(b, i, j):
                    effect[0, b, i, h, d] |= x != -INF
                    effect[1, b, i, h, d] |= x != INF
    out, lse, tol, lse_tol = plain_attend(q, k_pages, clean, table, p, t, sees, D ** -0.5)
    got, got_lse = beam.attend(q, k_pages, v_pages, table.cuda(), p.cuda(), t.cuda(), mask.cuda() if masked else None, return_lse=True)
    plus, minus = (torch.from_numpy(e).repeat_interleave(Hq // Hkv, dim=2) for e in effect)
    assert (plus | minus).any() and not (plus | minus).all()
    g = got.cpu().double()
    assert torch.equal(torch.isnan(g), plus & minus) and torch.equal(g == INF, plus & ~minus) and torch.equal(g == -INF, minus & ~plus)
    near(torch.where(plus | minus, 0.0, g), got_lse, (torch.where(plus | minus, 0.0, out), lse, tol, lse_tol))


def ragged_prompt(dtype, B, n, Hq, Hkv, D, page, fill):
    """Prompts of n / 4 to n tokens, all asked for as n: behind each is `fill`, or None: whatever bits."""
    lens = torch.linspace(n // 4, n, B).int()
    k_pages, _, table = a_cache(6, B, n, Hkv, D, page, dtype)
    k_pages = k_pages.contiguous()
    place = torch.full((len(k_pages), page), True)
    for b in range(B):
        for t in range(int(lens[b])):
            place[table[b, t // page], t % page] = False
    place = place[:, :, None, None].expand(k_pages.shape).cuda()
    if fill is None:
        bits = torch.randint(0, 256, (k_pages.numel() * k_pages.element_size(),), dtype=torch.uint8, generator=gen(7)).cuda().view(dtype).reshape(k_pages.shape)
        k_pages = torch.where(place, bits, k_pages)
    else:
        k_pages = k_pages.masked_fill(place, fill)
    q = torch.randn(B, n, Hq, D, generator=gen(8)).to(dtype).cuda()
    zero, whole = torch.zeros(B, dtype=torch.int32), torch.full((B,), n, dtype=torch.int32)
    return lens, (q, k_pages, k_pages, table.cuda(), zero.cuda(), whole.cuda())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (4, 1, 128)])
def test_attend_of_a_ragged_prompt_with_anything_behind_it(beam, dtype, Hq, Hkv, D):  # noqa: F811
    """The nodes of a sentence's own tokens come out bit for bit as where zeros lie behind them."""
    lens, args = ragged_prompt(dtype, 3, 200, Hq, Hkv, D, 16, 0.0)
    want, want_lse = beam.attend(*args, max_len=200, return_lse=True)
    assert torch.isfinite(want).all()
    for fill in (NAN, INF, -INF, None):
        _, other = ragged_prompt(dtype, 3, 200, Hq, Hkv, D, 16, fill)
        got, lse = beam.attend(*other, max_len=200, return_lse=True)
        for b in range(3):
            m = int(lens[b])
            assert torch.equal(got[b, :m], want[b, :m]) and torch.equal(lse[b, :m], want_lse[b, :m]), (fill, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_of_a_ragged_prompt_takes_no_longer_for_what_lies_behind_it(beam, dtype):  # noqa: F811
    """A tile of 64 tokens that holds such values takes a few times as long; a walk over its tokens for every element took 70 times."""
    times = {}
    for fill in (0.0, NAN, INF, None):
        _, args = ragged_prompt(dtype, 4, 400, 8, 2, 64, 16, fill)
        best = math.inf
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            beam.attend(*args, max_len=400)
            a.record()
            for _ in range(5):
                beam.attend(*args, max_len=400)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        times[fill] = best
    assert all(t <= 8 * times[0.0] for t in times.values()), times


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,n,Hq,Hkv,D,length", [(2, 5, 8, 4, 64, 400), (2, 16, 4, 2, 64, 300), (2, 16, 4, 2, 128, 300), (1, 1, 4, 4, 128, 6000), (2, 3, 6, 2, 80, 500), (2, 4, 8, 2, 256, 300),
                                                 (140, 2, 8, 8, 64, 40)])
def test_attend_of_few_rows_is_rounded_once(beam, dtype, B, n, Hq, Hkv, D, length):  # noqa: F811
    """Up to 32 rows a head (16 of 256): the weights' rounding does not show.  With u the type's half step, A = sum p |v| and e the scores' error (test_gpu_beam_ops.py):
    the result is off by u |o|, and a weight by u^2 of itself, 4 e, 2^-20 and the sum's L u32."""
    k_pages, v_pages, table = a_cache(1, B, length, Hkv, D, 16, dtype)
    q = torch.randn(B, n, Hq, D, generator=gen(2)).to(dtype).cuda()
    got = beam.attend(q, k_pages, v_pages, table.cuda(), torch.full((B,), length, dtype=torch.int32).cuda()).cpu().double()
    u, scale, kp, vp = U[dtype], D ** -0.5, k_pages.cpu(), v_pages.cpu()
    off = mean = 0.0
    for b in range(B):
        k, v = rows_of(kp, table, b, length), rows_of(vp, table, b, length)
        for h in range(Hq):
            x, kk, vv = q[b, :, h].cpu().double(), k[:, h * Hkv // Hq], v[:, h * Hkv // Hq]
            p = (x @ kk.T * scale).softmax(dim=1)
            want = p @ vv
            e = (D + 8) * U32 * (x.abs() @ kk.abs().T).amax(dim=1, keepdim=True) * scale
            tol = u * want.abs() + (p @ vv.abs()) * (u * u + 4 * e + 2.0 ** -20 + length * U32)
            assert ((got[b, :, h] - want).abs() <= tol).all(), float(((got[b, :, h] - want).abs() - tol).max())
            off, mean = off + float((got[b, :, h] - want).square().sum()), mean + float((want.to(dtype).double() - want).square().sum())
    assert off <= 1.05 ** 2 * mean                                      # as far from it as its own rounding


@pytest.mark.parametrize("B,heads", [(2000, 33), (2100, 64)])
def test_attend_in_more_workgroups_than_one_axis_takes(beam, B, heads):  # noqa: F811
    """One token a sentence and head, one or two heads a workgroup: more than 65536 of them."""
    D, page, most = 8, 16, 16
    lens = torch.randint(0, most + 1, (B,), generator=gen(1), dtype=torch.int32)
    pages = torch.randn(2, B, page, heads, D, generator=gen(2)).bfloat16()
    table = torch.randperm(B, generator=gen(3)).int()[:, None]
    q = torch.randn(B, 1, heads, D, generator=gen(4)).bfloat16()
    got, lse = beam.attend(q.cuda(), pages[0].cuda(), pages[1].cuda(), table.cuda(), lens.cuda(), return_lse=True)
    k, v = (p[table[:, 0].long()].double().transpose(1, 2) for p in pages)      # [B, heads, page, D]
    x = (k * q.double().transpose(1, 2)).sum(dim=3) * D ** -0.5
    x = x.masked_fill(torch.arange(page)[None, None] >= lens[:, None, None], -INF)
    want_lse = x.logsumexp(dim=2)
    p = (x - want_lse.clamp(min=-1e30)[..., None]).exp()
    want, room = (p[..., None] * v).sum(dim=2), (p[..., None] * v.abs()).sum(dim=2)
    e = (D + 8) * U32 * float((k.abs() * q.double().abs().transpose(1, 2)).sum(dim=3).max()) * D ** -0.5
    tol = U[torch.bfloat16] * want.abs() + room * (U[torch.bfloat16] + 4 * e + 2.0 ** -20 + most * U32)
    assert ((got[:, 0].cpu().double() - want).abs() <= tol).all()
    seen = want_lse > -INF
    assert torch.equal(lse[:, 0].cpu() > -INF, seen) and ((lse[:, 0].cpu().double() - want_lse)[seen].abs() <= 2 * e + 2.0 ** -20 + most * U32 + U32 * want_lse[seen].abs()).all()
