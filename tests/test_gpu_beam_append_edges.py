"""-m gpu: appending at the edges of what it accepts.  Tolerances are those of test_gpu_beam_ops.py."""
import pytest
import torch

from test_gpu_beam_ops import TYPES, U, a_cache, beam, gen, rotated  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
def test_positions_beyond_the_last_token(beam, dtype):  # noqa: F811
    """Tokens from 2^31 - 3 on: none has a place in the cache, and the queries are rotated by first + i all the same."""
    n, D, first = 6, 32, 2**31 - 3
    k_pages, v_pages, table = a_cache(1, 1, 64, 2, D, 16, dtype, fill=7.0)
    q, k = (torch.randn(1, n, 2, D, generator=gen(s)).to(dtype) for s in (2, 3))
    inv = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float()
    got = beam.append(k.cuda(), k.cuda(), k_pages, v_pages, table.cuda(), torch.tensor([first], dtype=torch.int32).cuda(), inv_freq=inv.cuda(), q=q.cuda())
    want, tol = rotated(q[0].double(), first + torch.arange(n, dtype=torch.int64), inv, False)
    assert ((got[0].cpu().double() - want).abs() <= U[dtype] * want.abs() + tol * (1 + U[dtype])).all()
    assert (k_pages == 7).all() and (v_pages == 7).all()
