"""-m gpu: selection from logits whose rows hold masks' fill values of any size, and from equal rows wherever they lie in memory.

Tolerances are those of test_gpu_beam_ops.py: the score's rounding and 2^-22 for the exponentials.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_beam_ops import TYPES, U32, beam, check_select, gen, plain_select  # noqa: F401

pytestmark = pytest.mark.gpu


def around(x):
    """x and its neighbours in fp32."""
    return [float(np.nextafter(np.float32(x), np.float32(to))) for to in (-np.inf, np.inf)] + [float(x)]


FILLS = [-1e4, -65504.0, 1e9, -1e9, 1e10, -1e10, -1e18, 1e18, -1e20, -1e30, 1e30, 1e36, -1e36] + [
    s * x for e in (2.0 ** 10, 2.0 ** 20, 2.0 ** 24, 2.0 ** 30, 1e37) for x in around(e) for s in (1, -1)]
V = 41000                                              # several parts of a row in every type


def filled(dtype):
    """A sentence for each fill value that the type holds: a row of nothing else; a row whose only other logits lie in its last part; a
    row around the fill's size, of which the first half is nothing but that."""
    fills = torch.tensor(FILLS, dtype=torch.float64).to(dtype)
    fills = fills[torch.isfinite(fills)]
    B, g = len(fills), gen(11)
    x = fills[:, None, None].expand(B, 3, V).clone()
    x[:, 1, V - 300:] = (torch.randn(B, 300, generator=g) * 2).to(dtype)
    some = fills.double()[:, None] * torch.randint(4, 9, (B, V), generator=g) / 8
    x[:, 2] = some.to(dtype)
    x[:, 2, V // 2:] = torch.where(torch.rand(B, V - V // 2, generator=g) < 0.5, x[:, 2, V // 2:], (torch.randn(B, V - V // 2, generator=g) * 2).to(dtype))
    score = torch.tensor([0.3, -4.5, -2.1])[None] - torch.rand(B, 3, generator=g)
    return x, score


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k_out", [1, 6, 64])
def test_select_from_rows_of_fill_values(beam, dtype, k_out):  # noqa: F811
    logits, score = filled(dtype)
    check_select(beam, logits, score, None, k_out)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_row_of_fill_values_is_lost(beam, dtype):  # noqa: F811
    """Every row by itself: its normaliser is finite, so k_out extensions come back."""
    logits, score = filled(dtype)
    one = logits.reshape(-1, 1, V)
    got = [x.cpu() for x in beam.select(one.cuda(), score.reshape(-1, 1).cuda(), None, 4, 2, 0)]
    assert (got[1] == 0).all() and (got[3] & 2 == 0).all()
    want = plain_select(one, score.reshape(-1, 1), None, 4)[2]
    near = np.abs(want) < 1e30
    assert (np.abs(got[2].numpy() - want)[near] <= np.abs(want)[near] * U32 + 2.0 ** -22).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,k,k_out", [(9, 4, 4), (777, 5, 10), (1001, 64, 64), (32003, 7, 7), (50001, 5, 5), (50002, 6, 24)])
def test_equal_rows_go_by_their_order(beam, dtype, V, k, k_out):  # noqa: F811
    """Rows alike in logits and score, which start at different offsets from 16 bytes: equal extensions come in the order of the rows."""
    logits = (torch.randn(6, 1, V, generator=gen(V)) * 2).to(dtype).expand(6, k, V).contiguous()
    score = (-torch.rand(6, 1, generator=gen(k)) - 3).expand(6, k).contiguous()
    check_select(beam, logits, score, None, k_out)
    for lead, ld in ((1, V + 2), (3, V + 5)):
        room = torch.full((6, k, ld + lead), math.nan, dtype=dtype)
        room[:, :, lead:lead + V] = logits
        check_select(beam, logits, score, None, k_out, room.cuda()[:, :, lead:lead + V])


def best_of_many(logits, score, k_out):
    """(token, backptr, score) of one sentence in 64 bits, without a sort of everything."""
    x = logits.double()
    s = (torch.log_softmax(x, dim=1) + score.double()[:, None]).flatten().numpy()
    at = np.nonzero(s >= np.partition(s, len(s) - k_out)[len(s) - k_out])[0]
    at = at[np.lexsort((at, -s[at]))][:k_out]
    return at % logits.shape[1], at // logits.shape[1], s[at]


@pytest.mark.parametrize("k_out", [1, 40, 64])
def test_select_from_more_parts_than_the_second_launch_holds(beam, k_out):  # noqa: F811
    """64 rows of 17 parts; in the second sentence every part has the same best, and most rows are equal."""
    k, V = 64, 152000
    logits = torch.randn(2, k, V, generator=gen(1)) * 2
    logits[1] = -1.0
    logits[1, :, ::1000] = 3.0
    score = -torch.rand(2, k, generator=gen(2)) * 4 - 5
    score[1] = -5.0
    score[1, :6] = -9.0
    got = [x.cpu().numpy() for x in beam.select(logits.cuda(), score.cuda(), None, k_out, 2, 0)]
    for b in range(2):
        token, back, s = best_of_many(logits[b], score[b], k_out)
        assert np.array_equal(got[0][b], token) and np.array_equal(got[1][b], back), b
        assert (np.abs(got[2][b] - s) <= np.abs(s) * U32 + 2.0 ** -22).all()
        assert np.array_equal(got[3][b], (token == 2).astype(np.uint8))
