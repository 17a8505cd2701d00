"""-m "not gpu": the operators around a long cache refuse what they cannot do, before the device is touched."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_1804_06609_amd as dba
from paper_1804_06609_amd import beam
from test_beam_ops_cpu import AT, BAD_CACHES, _cache, _heads, _refused

HERE = os.path.dirname(os.path.abspath(__file__))
R = ctypes.byref
K, V, Q, O = (AT + i * (1 << 26) for i in range(1, 5))      # places apart from each other and from AT
FAR = AT + (1 << 40)


def test_the_struct_of_norms_is_laid_out_as_in_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    (tmp_path / "x.c").write_text('#include "dba_beam.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu\\n", sizeof(dba_norms), '
                                  'offsetof(dba_norms, format), offsetof(dba_norms, eps)); return 0; }\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(os.path.dirname(HERE), "include"), str(tmp_path / "x.c"), "-o", str(tmp_path / "x")], check=True)
    out = subprocess.run([str(tmp_path / "x")], capture_output=True, text=True, check=True).stdout
    assert out.split() == [str(x) for x in (ctypes.sizeof(beam._Norms), beam._Norms.format.offset, beam._Norms.eps.offset)]
    assert len(beam._pack_norms(0, 0, 0, 0, 0, 1.0)) == ctypes.sizeof(beam._Norms)


# ---- appending -------------------------------------------------------------------------------------------------------
def _norms(qw=FAR, kw=FAR, qs=64, ks=64, fmt=2, eps=1e-6):
    return beam._Norms(qw, kw, qs, ks, fmt, eps)


def _append(cache=None, k=None, v=None, q=None, q_out=None, q_heads=8, B=2, n=3, norms=None, first=AT, count=None, position=AT, axes=1, axis=None, inv=AT, rot=64):
    return beam.load().dba_cache_append_normed(B, n, R(cache or _cache()), R(k or _heads(K)), R(v or _heads(V)), q_heads, R(q) if q else None, R(q_out) if q_out else None,
                                               R(norms) if norms else None, first, count, position, axes, axis, inv, rot, 0, None)


@pytest.mark.parametrize("kw,frag", BAD_CACHES)
def test_append_refuses_a_cache(kw, frag):
    _refused(_append(_cache(**kw)), frag)


@pytest.mark.parametrize("kw,frag", [
    (dict(B=0), "B"), (dict(n=0), "n"), (dict(n=(1 << 22) + 1), "n"), (dict(first=None), "first"), (dict(inv=None), "inv_freq"), (dict(rot=8), "rot_dim"),
    (dict(rot=80), "rot_dim"), (dict(rot=-16), "rot_dim"), (dict(k=_heads(data=None)), "NULL"), (dict(v=_heads(V, t=4)), "16 bytes"),
    (dict(q=_heads(Q)), "together"), (dict(q_out=_heads(Q)), "together"), (dict(q=_heads(Q), q_out=_heads(O), q_heads=0), "q_heads"),
    (dict(q=_heads(Q), q_out=_heads(Q, t=2048)), "two sets"), (dict(q=_heads(Q), q_out=_heads(O + 4)), "16 bytes"),
    (dict(axes=0, axis=AT), "axes"), (dict(axes=65537, axis=AT), "axes"), (dict(axes=3), "axis_dev"), (dict(axes=3, axis=AT, position=None), "position_dev"),
    (dict(norms=_norms(eps=0.0)), "eps"), (dict(norms=_norms(eps=float("nan"))), "eps"), (dict(norms=_norms(eps=float("inf"))), "eps"), (dict(norms=_norms(eps=-1.0)), "eps"),
    (dict(norms=_norms(fmt=1)), "fp32"), (dict(norms=_norms(fmt=5)), "fp32"), (dict(norms=_norms(qw=FAR + 8)), "16 bytes"), (dict(norms=_norms(ks=4)), "16 bytes"),
    (dict(norms=_norms(qs=-64)), "16 bytes"), (dict(norms=_norms(fmt=0, ks=2)), "16 bytes"),
    (dict(q=_heads(Q), q_out=_heads(K)), "overlaps k"), (dict(q=_heads(Q), q_out=_heads(Q + 64)), "overlaps"), (dict(q=_heads(Q), q_out=_heads(O, t=64)), "pieces"),
    (dict(q=_heads(Q), q_out=_heads(O), first=O + 4), "counts"), (dict(q=_heads(Q), q_out=_heads(O), position=O + 64), "counts"), (dict(q=_heads(Q), q_out=_heads(O), inv=O), "counts"),
    (dict(q=_heads(Q), q_out=_heads(O), axes=2, axis=O), "counts"), (dict(q=_heads(Q), q_out=_heads(O), count=O), "counts"),
    (dict(q=_heads(Q), q_out=_heads(O), norms=_norms(qw=O + 512)), "weights"), (dict(q=_heads(Q), q_out=_heads(O), norms=_norms(kw=O - 256)), "weights"),
])
def test_append_refuses(kw, frag):
    _refused(_append(**kw), frag)


# ---- attention behind a common prefix --------------------------------------------------------------------------------
def _shared(cache=None, q=None, out=None, q_heads=8, B=2, n=3, shared=AT, pages=4, shared_len=AT, max_shared=64, prefix=AT, tree=AT, mask=AT, words=1, max_len=128, scale=0.125,
            lse=None, ws=FAR, nbytes=1 << 40):
    return beam.load().dba_shared_attend(B, n, q_heads, R(q or _heads(Q)), R(cache or _cache()), shared, pages, shared_len, max_shared, prefix, tree, mask, words, max_len, scale,
                                         R(out or _heads(O)), lse, ws, nbytes, None)


@pytest.mark.parametrize("kw,frag", BAD_CACHES)
def test_shared_refuses_a_cache(kw, frag):
    _refused(_shared(_cache(**kw)), frag)


@pytest.mark.parametrize("kw,frag", [
    (dict(B=0), "B"), (dict(B=65536), "B"), (dict(n=0), "n"), (dict(n=1 << 21), "n"), (dict(q_heads=6), "multiple"), (dict(q_heads=0), "q_heads"),
    (dict(B=60000, n=1 << 8), "2^26"), (dict(pages=0), "shared_pages"), (dict(pages=1 << 27), "shared_pages"), (dict(max_shared=0), "max_shared"), (dict(max_shared=65), "max_shared"),
    (dict(shared=None), "NULL"), (dict(shared_len=None), "NULL"), (dict(prefix=None), "NULL"), (dict(tree=None), "mask"), (dict(words=-1), "mask"),
    (dict(max_len=0), "max_len"), (dict(max_len=129), "max_len"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(q=_heads(data=None)), "NULL"), (dict(out=_heads(O + 8)), "16 bytes"), (dict(ws=None), "256"), (dict(ws=FAR + 128), "256"),
    (dict(out=_heads(Q + 64)), "part of q"), (dict(out=_heads(O, t=64)), "pieces"), (dict(lse=O + 4), "out_lse_dev"), (dict(lse=Q), "out_lse_dev"), (dict(ws=Q), "workspace"), (dict(ws=O), "workspace"),
    (dict(lse=FAR + 64), "workspace"),
])
def test_shared_refuses(kw, frag):
    _refused(_shared(**kw), frag)


def test_shared_workspace():
    size = beam.load().dba_shared_attend_workspace_bytes
    need = size(2, 3, 8, R(_cache()), 4, 64, 128)
    assert 0 < need < 1 << 24
    _refused(_shared(nbytes=need - 1), "workspace", dba.DBA_ENOMEM)
    for bad in [(0, 3, 8, 4, 64, 128), (2, 3, 8, 0, 64, 128), (2, 3, 8, 4, 65, 128), (2, 3, 7, 4, 64, 128), (2, 3, 8, 4, 64, 129)]:
        assert size(bad[0], bad[1], bad[2], R(_cache()), *bad[3:]) == 0
    assert size(2, 3, 8, None, 4, 64, 128) == 0
    assert size(65535, 128, 8, R(_cache()), 4, 64, 128) > 1 << 35


# ---- weighing --------------------------------------------------------------------------------------------------------
def _weigh(cache=None, q=None, q_heads=8, B=2, n=3, lse=AT, prefix=AT, tree=AT, mask=AT, words=1, count=None, max_len=128, scale=0.125, by_head=1, score=K, ss=1024, sh=256,
           out=V, os_=1024, oh=256, width=200, ws=FAR, nbytes=1 << 30):
    return beam.load().dba_cache_weigh(B, n, q_heads, R(q or _heads(Q)), lse, R(cache or _cache()), prefix, tree, mask, words, count, max_len, scale, by_head, score, ss, sh, out, os_, oh, width, ws, nbytes, None)


@pytest.mark.parametrize("kw,frag", BAD_CACHES)
def test_weigh_refuses_a_cache(kw, frag):
    _refused(_weigh(_cache(**kw)), frag)


@pytest.mark.parametrize("kw,frag", [
    (dict(B=0), "B"), (dict(n=0), "n"), (dict(n=1 << 21), "n"), (dict(q_heads=6), "multiple"), (dict(lse=None), "lse_dev"), (dict(lse=AT + 2), "lse_dev"), (dict(prefix=None), "prefix_dev"),
    (dict(tree=None), "mask"), (dict(words=-1), "mask"), (dict(max_len=0), "max_len"), (dict(max_len=129), "max_len"), (dict(scale=float("nan")), "scale"),
    (dict(score=None), "NULL"), (dict(out=None), "NULL"), (dict(score=K + 2), "4 bytes"), (dict(oh=-1), "negative"), (dict(width=127), "width"), (dict(width=(1 << 28) + 1), "width"),
    (dict(out=K, oh=200), "two sets"), (dict(out=K, os_=2048), "two sets"), (dict(out=K + 4), "overlaps"), (dict(oh=199), "rows"), (dict(out=Q), "lies in"), (dict(out=AT), "lies in"),
    (dict(lse=V + 400), "lies in"), (dict(mask=V + 1024), "lies in"), (dict(q=_heads(data=None)), "NULL"), (dict(cache=_cache(k=V - 4096)), "the cache"),
])
def test_weigh_refuses(kw, frag):
    _refused(_weigh(**kw), frag)


def test_weigh_workspace():
    size = beam.load().dba_cache_weigh_workspace_bytes
    need = size(2, 3, 8, R(_cache()), 0, 128)
    assert 0 < need < 1 << 20 and size(2, 3, 8, R(_cache()), 1, 128) == 0 and size(2, 3, 8, R(_cache(heads=1)), 0, 128) == 0
    one = dict(by_head=0, sh=0, oh=0)
    _refused(_weigh(nbytes=need - 1, **one), "workspace", dba.DBA_ENOMEM)
    for kw in (dict(ws=None), dict(ws=FAR + 64)):
        _refused(_weigh(**kw, **one), "256")
    for kw in (dict(ws=K), dict(ws=V), dict(ws=Q), dict(lse=FAR)):
        _refused(_weigh(**kw, **one), "in the workspace")
    for bad in [(0, 3, 8, 0, 128), (2, 3, 8, 0, 129), (2, 3, 7, 0, 128)]:
        assert size(bad[0], bad[1], bad[2], R(_cache()), *bad[3:]) == 0


# ---- eviction --------------------------------------------------------------------------------------------------------
def _evict(cache=None, B=2, new_table=AT + 4096, stride=8, pages=8, by_head=1, score=K, ss=1024, sh=256, prefix=AT, tree=AT, keep=10, budget=None, sinks=0, recent=0, max_len=128,
           new_prefix=O, new=V, ns=1024, nh=256, width=200, ws=FAR, nbytes=1 << 30):
    return beam.load().dba_cache_evict(B, R(cache or _cache()), new_table, stride, pages, by_head, score, ss, sh, prefix, tree, keep, budget, sinks, recent, max_len, new_prefix,
                                       new, ns, nh, width, ws, nbytes, None)


@pytest.mark.parametrize("kw,frag", BAD_CACHES)
def test_evict_refuses_a_cache(kw, frag):
    _refused(_evict(_cache(**kw)), frag)


@pytest.mark.parametrize("kw,frag", [
    (dict(B=0), "B"), (dict(B=65536), "B"), (dict(keep=0), "keep"), (dict(max_len=0), "max_len"), (dict(max_len=129), "max_len"), (dict(score=None), "NULL"), (dict(score=K + 1), "4 bytes"),
    (dict(nh=-4), "negative"), (dict(new_table=None), "NULL"), (dict(prefix=None), "NULL"), (dict(new_prefix=None), "NULL"), (dict(pages=0), "new_max_pages"), (dict(stride=7), "new_max_pages"),
    (dict(pages=1 << 27, stride=1 << 27), "new_max_pages"), (dict(sinks=-1), "sinks"), (dict(recent=-1), "recent"), (dict(width=127), "width"), (dict(width=(1 << 28) + 1), "width"),
    (dict(ws=None), "256"), (dict(ws=FAR + 64), "256"), (dict(cache=_cache(token_stride=64)), "overlap"), (dict(nh=199), "rows"), (dict(new=K), "what is read"), (dict(new=K + 4), "what is read"),
    (dict(new_prefix=V + 4), "overlap"), (dict(new_prefix=AT + 4), "what is read"), (dict(new_prefix=AT + 4096), "what is read"), (dict(ws=K), "what is read"), (dict(ws=V), "overlap"),
    (dict(budget=O), "what is read"), (dict(new_prefix=FAR), "overlap"), (dict(cache=_cache(k=V - 4096)), "in the cache"), (dict(cache=_cache(v=K)), "in the cache"),
    (dict(cache=_cache(v=FAR)), "in the cache"), (dict(cache=_cache(k=O - 64)), "in the cache"),
])
def test_evict_refuses(kw, frag):
    _refused(_evict(**kw), frag)


def test_evict_workspace():
    size = beam.load().dba_cache_evict_workspace_bytes
    need = size(2, R(_cache()), 1, 10, 128)
    assert 0 < need < 1 << 20 and size(2, R(_cache()), 0, 10, 128) <= need and size(2, R(_cache()), 1, 2**31 - 1, 128) < 1 << 20
    _refused(_evict(nbytes=need - 1), "workspace", dba.DBA_ENOMEM)
    for bad in [(0, 10, 128), (2, 0, 128), (2, 10, 0), (2, 10, 129)]:
        assert size(bad[0], R(_cache()), 1, *bad[1:]) == 0
    assert size(2, None, 1, 10, 128) == 0


# ---- the binding -----------------------------------------------------------------------------------------------------
def test_tensors_have_to_be_on_the_gpu():
    x, pages, table, one = torch.zeros(1, 2, 4, 16), torch.zeros(3, 8, 4, 16), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(dba.DbaError, match="GPU"):
        beam.append(x, x, pages, pages, table, one, eps=1e-6)
    with pytest.raises(dba.DbaError, match="GPU"):
        beam.attend_shared(x, pages, pages, table[0], one, table, one)
    with pytest.raises(dba.DbaError, match="GPU"):
        beam.weigh(torch.zeros(1, 4, 16), x, torch.zeros(1, 2, 4), pages, table, one)
    with pytest.raises(dba.DbaError, match="GPU"):
        beam.evict(torch.zeros(1, 4, 16), pages, pages, table, table, one, keep=3)


def test_what_requires_a_gradient_is_refused():
    x, pages, table, one = torch.zeros(1, 2, 4, 16), torch.zeros(3, 8, 4, 16), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    grad = lambda t: t.clone().requires_grad_()
    calls = [lambda: beam.append(x, x, pages, pages, table, one, eps=1e-6, k_weight=grad(torch.ones(16))),
             lambda: beam.append(grad(x), x, pages, pages, table, one, eps=1e-6),
             lambda: beam.attend_shared(grad(x), pages, pages, table[0], one, table, one),
             lambda: beam.attend_shared(x, grad(pages), pages, table[0], one, table, one),
             lambda: beam.weigh(grad(torch.zeros(1, 4, 16)), x, torch.zeros(1, 2, 4), pages, table, one),
             lambda: beam.weigh(torch.zeros(1, 4, 16), x, grad(torch.zeros(1, 2, 4)), pages, table, one),
             lambda: beam.evict(grad(torch.zeros(1, 4, 16)), pages, pages, table, table, one, keep=3)]
    for call in calls:
        with pytest.raises(dba.DbaError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(dba.DbaError, match="GPU"):
            call()
