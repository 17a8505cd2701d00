"""-m gpu: attention behind a common prefix: what its weights' rounding leaves."""
import pytest
import torch

from test_gpu_beam_ops import U, U32, beam, gen  # noqa: F401
from test_gpu_cache_ops import cuda, ints, setting, tokens_of

pytestmark = pytest.mark.gpu
HALVES = [torch.float16, torch.bfloat16]


# B, n, Hq, Hkv, D, page, common, own: rows a head behind the common tokens B n Hq / Hkv, behind a sentence's own n Hq / Hkv
ROUNDED = [
    (5, 20, 8, 2, 128, 16, 700, 90), (6, 5, 16, 2, 64, 32, 900, 70), (3, 16, 8, 2, 80, 64, 400, 150), (2, 40, 8, 2, 128, 16, 60, 700),    # the kernel for many rows; own ones: shared tiles, 40, 64, 160
    (5, 20, 8, 2, 128, 8, 500, 90), (4, 9, 8, 2, 64, 8, 600, 200), (4, 6, 8, 2, 256, 16, 400, 60),                                         # shared tiles for either kind
    (2, 12, 8, 2, 128, 16, 500, 100), (1, 50, 4, 4, 64, 16, 300, 120), (3, 2, 4, 2, 128, 16, 800, 40),                                     # up to 64 and up to 32 rows
]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("B,n,Hq,Hkv,D,page,common,own", ROUNDED)
def test_shared_is_rounded_once(beam, dtype, B, n, Hq, Hkv, D, page, common, own):  # noqa: F811
    """The weights' rounding does not show, however many rows there are.  With u the type's half step, A = sum p |v| and e the scores' error (test_gpu_beam_ops.py): the result is off by u |o|,
    and a weight by u^2 of itself, 4 e, 2^-20 and the sum's L u32; on the whole the result is as far off as its own rounding."""
    k_pages, v_pages, shared, table = setting(dtype, B, Hkv, D, page, common, [own] * B, [0] * B)
    q = torch.randn(B, n, Hq, D, generator=gen(2)).to(dtype).cuda()
    got = beam.attend_shared(q, k_pages, v_pages, *cuda(shared, ints(common), table, ints(*[own] * B))).cpu().double()
    u, scale, kp, vp = U[dtype], D ** -0.5, k_pages.cpu().double().reshape(-1, Hkv, D), v_pages.cpu().double().reshape(-1, Hkv, D)
    first = tokens_of(shared, len(k_pages), page, common)[1]
    off = mean = 0.0
    for b in range(B):
        at = torch.cat((first, tokens_of(table[b], len(k_pages), page, own)[1]))
        for h in range(Hq):
            x, kk, vv = q[b, :, h].cpu().double(), kp[at, h * Hkv // Hq], vp[at, h * Hkv // Hq]
            p = (x @ kk.T * scale).softmax(dim=1)
            want = p @ vv
            e = (D + 8) * U32 * (x.abs() @ kk.abs().T).amax(dim=1, keepdim=True) * scale
            tol = u * want.abs() + (p @ vv.abs()) * (u * u + 4 * e + 2.0 ** -20 + (common + own) * U32)
            assert ((got[b, :, h] - want).abs() <= tol).all(), float(((got[b, :, h] - want).abs() - tol).max())
            off, mean = off + float((got[b, :, h] - want).square().sum()), mean + float((want.to(dtype).double() - want).square().sum())
    assert off <= 1.05 ** 2 * mean, (off / mean) ** 0.5
