"""-m gpu: reordering of states that are views of one tensor."""
import pytest
import torch

from test_gpu_beam_ops import beam, gen, plain_reorder  # noqa: F401

pytestmark = pytest.mark.gpu


def test_reorder_of_views_that_interleave(beam):  # noqa: F811
    """Keys beside values in one tensor, in place; from one half of a tensor into the other; halves of a record of uneven widths."""
    B, k = 3, 6
    back = torch.randint(-1, k, (B, k), generator=gen(1), dtype=torch.int32)
    kv = torch.randn(B, k, 4, 2, 16, generator=gen(2))
    want = plain_reorder(back, kv)
    dev = kv.cuda()
    beam.reorder(back.cuda(), [dev[:, :, :, 0], dev[:, :, :, 1]])
    assert torch.equal(dev.cpu(), want)
    both = kv.cuda()
    beam.reorder(back.cuda(), [both[:, :, :, 0]], [both[:, :, :, 1]])
    assert torch.equal(both[:, :, :, 0].cpu(), kv[:, :, :, 0]) and torch.equal(both[:, :, :, 1].cpu(), want[:, :, :, 0])
    record = torch.randn(B, k, 37, generator=gen(3))
    dev = record.cuda()
    beam.reorder(back.cuda(), [dev[:, :, :30], dev[:, :, 30:]])
    assert torch.equal(dev.cpu(), plain_reorder(back, record))


def test_reorder_refuses_tensors_that_share_memory(beam):  # noqa: F811
    from paper_1804_06609_amd import DbaError
    back = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    a, b = torch.randn(2, 4, 5, device="cuda"), torch.randn(2, 4, 5, device="cuda")
    kept = a.clone(), b.clone()
    for states, out in (([a, a], None), ([a, b], [b, a]), ([a, b], [b, b]), ([a, a[:, :, 2:]], None)):
        with pytest.raises(DbaError, match="overlap"):
            beam.reorder(back, states, out)
    with pytest.raises(DbaError, match="backptr"):
        beam.reorder(back, [back])
    assert torch.equal(a, kept[0]) and torch.equal(b, kept[1])
