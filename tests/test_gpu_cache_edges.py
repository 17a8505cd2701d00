"""-m gpu: the operators around a long cache where many rows go through kernels of their own: attention behind a common prefix of more than 64 rows a head (in 16 bits, heads of up to 128, pages of 16 tokens at
least), and weighing of more than 128.  Pages that are not there, places that nobody sees, pools beyond 2^31 elements; counts, scales and ends.  Tolerances as in test_gpu_cache_ops.py."""
import math

import pytest
import torch

from test_gpu_beam_ops import TYPES, beam, gen  # noqa: F401
from test_gpu_cache_ops import check_shared, check_weigh, cuda, ints, setting

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf
# B, n, Hq, Hkv, D, page: 80 to 160 rows a head
MANY = [(20, 8, 4, 2, 128, 16), (16, 5, 8, 8, 64, 64), (9, 11, 8, 2, 80, 32)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,n,Hq,Hkv,D,page", MANY)
@pytest.mark.parametrize("common", [5, 100, 333])
def test_shared_many_rows_and_pages_that_are_not_there(beam, dtype, B, n, Hq, Hkv, D, page, common):  # noqa: F811
    def some(k_pages, v_pages, shared, table):
        if len(shared) > 1:
            shared[len(shared) // 2] = -1
        shared[-1], table[0, 0], table[B - 1, -1] = 2**31 - 1, -2**31, -1
    check_shared(beam, dtype, B, n, Hq, Hkv, D, page, common, [40] * B, [n] * B, masked=False, spoil=some)
    check_shared(beam, dtype, B, n, Hq, Hkv, D, page, common, [40] * B, [n] * B, masked=True, spoil=some, max_shared=max(1, common - 3) if common < 100 else None)

    k_pages, v_pages, shared, table = setting(dtype, B, Hkv, D, page, common, [30] * B, [0] * B)
    shared[:], table[0] = -1, -5
    q = torch.randn(B, n, Hq, D, generator=gen(1)).to(dtype).cuda()
    out, lse = beam.attend_shared(q, k_pages, v_pages, *cuda(shared, ints(common), table, ints(*[30] * B)), return_lse=True)
    assert (out[0] == 0).all() and (lse[0] == -INF).all() and torch.isfinite(lse[1:]).all() and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,n,Hq,Hkv,D,page", MANY)
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_shared_many_rows_and_values_that_are_not_finite(beam, dtype, B, n, Hq, Hkv, D, page, bad):  # noqa: F811
    """Behind the end, in pages that nobody has and in masked places they do not matter; an element of a common token that is not finite reaches that element of all, and a key all of them at the most."""
    common = 2 * page + 5
    k_pages, v_pages, shared, table = setting(dtype, B, Hkv, D, page, common, [40] * B, [n + page] * B)      # (more room than is used)
    absent = int(shared[1])
    shared[1] = -7
    q = torch.randn(B, n, Hq, D, generator=gen(1)).to(dtype).cuda()
    mask = torch.zeros(B, n, 1, dtype=torch.int64)
    mask[:, :, 0] = ~torch.tensor(4)                                    # nobody sees token 2 of the tree
    args = cuda(shared, ints(common), table, ints(*[20] * B), ints(*[n] * B), mask)
    want = beam.attend_shared(q, k_pages, v_pages, *args, return_lse=True)
    assert torch.isfinite(want[0]).all() and torch.isfinite(want[1]).all()
    for x in (k_pages, v_pages):
        x[int(shared[-1]), common % page:] = bad
        x[absent] = bad
        for b in range(B):
            x[int(table[b, 22 // page]), 22 % page] = bad
            x[int(table[b, (20 + n) // page]), (20 + n) % page:] = bad
    got = beam.attend_shared(q, k_pages, v_pages, *args, return_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    v_pages[int(shared[0]), 3, Hkv - 1, 7] = bad
    got = beam.attend_shared(q, k_pages, v_pages, *args)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[:, :, Hq - Hq // Hkv:, 7] = True
    assert torch.equal(~torch.isfinite(got), hit) and torch.equal(got[~hit], want[0][~hit])
    k_pages[int(shared[0]), 2, Hkv - 1, 0] = bad
    got = beam.attend_shared(q, k_pages, v_pages, *args)
    assert torch.equal(got[:, :, :Hq - Hq // Hkv], want[0][:, :, :Hq - Hq // Hkv])      # (heads of the other keys)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,n,Hq,Hkv,D,page", MANY)
def test_shared_many_rows_twice_is_the_same(beam, dtype, B, n, Hq, Hkv, D, page):  # noqa: F811
    k_pages, v_pages, shared, table = setting(dtype, B, Hkv, D, page, 3000, [40] * B, [n] * B)
    q = torch.randn(B, n, Hq, D, generator=gen(1)).to(dtype).cuda()
    args = cuda(shared, ints(3000), table, ints(*[40] * B), ints(*[n] * B))
    want = beam.attend_shared(q, k_pages, v_pages, *args, return_lse=True)
    for _ in range(20):
        got = beam.attend_shared(q, k_pages, v_pages, *args, return_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("page", [16, 1024])
def test_shared_many_rows_and_offsets_beyond_32_bits(beam, dtype, page):  # noqa: F811
    """A pool of 4 GiB and more: the last pages lie behind 2^31 elements."""
    H, D, B = 8, 128, 45
    n = (1 << 31) // (page * H * D) + 40
    pool = torch.empty((n, page, H, D), dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    last = [n - 1, n - 7, 0, n - 9, n - 11]
    for p in last:
        pool[p].normal_(generator=g)
    small = torch.stack([pool[p] for p in last])
    q = torch.randn(B, 2, H, D, generator=gen(1)).to(dtype).cuda()      # 90 rows a head
    results = []
    for where, ids in ((pool, last), (small, range(5))):
        ids = ints(*ids)
        results.append(beam.attend_shared(q, where, where, *cuda(ids[:3], ints(2 * page + 9), ids[2:].repeat(B, 1), ints(*[page + 3, 1, 2 * page - 1] * (B // 3))), return_lse=True))
    assert all(torch.equal(x, y) for x, y in zip(*results)) and torch.isfinite(results[0][0]).all()


# rows that are split over workgroups, in sentences of several and of one: B, n, Hq, Hkv, D, page, prefix, tree
ROWS = [(2, 80, 8, 2, 64, 16, [100, 30], [90, 80]), (3, 300, 4, 2, 128, 32, [0, 500, 20], [300, 10, 330]), (2, 150, 6, 3, 40, 8, [77, 0], [150, 200])]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("by_head", [True, False])
@pytest.mark.parametrize("shape", ROWS)
def test_weigh_many_rows_counts_scales_and_ends(beam, dtype, by_head, shape):  # noqa: F811
    """Counts that end in front of a later split's rows, at its first one, and of no row."""
    B, n = shape[:2]
    for masked in (False, True):
        check_weigh(beam, dtype, *shape, masked=masked, by_head=by_head, count=([3, n, -1] * B)[:B])
        check_weigh(beam, dtype, *shape, masked=masked, by_head=by_head, count=([0, 32, n + 5] * B)[:B], scale=-0.2)
        check_weigh(beam, dtype, *shape, masked=masked, by_head=by_head, count=([64, n - 1, 1] * B)[:B], scale=0.0)
        for max_len in (1, 64, 130):
            check_weigh(beam, dtype, *shape, masked=masked, by_head=by_head, max_len=max_len)
