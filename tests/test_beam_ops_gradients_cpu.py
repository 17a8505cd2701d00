"""-m "not gpu": the operators have no gradient, and say so where torch would record one."""
import pytest
import torch

from paper_1804_06609_amd import DbaError, beam


def calls():
    B, k, V, H, D = 1, 2, 8, 2, 16
    z = torch.zeros
    back, first = z(B, k, dtype=torch.int32), z(B, dtype=torch.int32)
    pages, table, x = z(3, 4, H, D), z(B, 2, dtype=torch.int32), z(B, k, H, D)
    new = lambda t: t.clone()
    return {
        "select": (lambda a: beam.select(a[0], a[1], None, 2, 2, 0), [z(B, k, V), z(B, k)]),
        "reorder": (lambda a: beam.reorder(back, a), [z(B, k, 3), z(B, k, 4)]),
        "append": (lambda a: beam.append(a[0], a[1], new(pages), new(pages), table, first, inv_freq=a[2], q=a[3]), [new(x), new(x), z(D // 2), new(x)]),
        "attend": (lambda a: beam.attend(a[0], a[1], a[2], table, first), [new(x), new(pages), new(pages)]),
    }


@pytest.mark.parametrize("name,which", [(n, i) for n, (_, a) in calls().items() for i in range(len(a))])
def test_a_gradient_is_refused(name, which):
    call, args = calls()[name]
    args[which].requires_grad_()
    with pytest.raises(DbaError, match="no gradient"):
        call(args)
    with torch.no_grad(), pytest.raises(DbaError, match="GPU"):          # as without one
        call(args)


@pytest.mark.parametrize("name", list(calls()))
def test_without_one_it_is_not(name):
    call, args = calls()[name]
    with pytest.raises(DbaError, match="GPU"):
        call(args)
