"""-m gpu: attention over a tree at the edges of what it accepts.  Tolerances are those of test_gpu_beam_ops.py."""
import pytest
import torch

from test_gpu_beam_ops import TYPES, a_cache, beam, gen, near, plain_attend  # noqa: F401

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
