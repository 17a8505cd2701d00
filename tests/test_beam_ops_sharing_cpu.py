"""-m "not gpu": calls of the operators whose tensors share memory that is written are refused before the device is touched."""
import ctypes

import pytest

from paper_1804_06609_amd import beam
from test_beam_ops_cpu import AT, _append, _cache, _heads, _refused, _reorder, _select, _state

MB = 1 << 20
FAR = AT + 64 * MB


# 2 x 8 rows of 512 bytes: 8 KB
@pytest.mark.parametrize("states,frag", [
    ([_state(dst=FAR, src=FAR), _state(dst=FAR, src=FAR)], "states 0 and 1"),                                     # one state twice, in place
    ([_state(dst=FAR, src=FAR + MB), _state(dst=FAR + MB, src=FAR)], "states 0 and 1"),                           # swapped buffers
    ([_state(dst=FAR, src=FAR + MB), _state(dst=FAR, src=FAR + 2 * MB)], "states 0 and 1"),                       # one place for two
    ([_state(dst=FAR, src=FAR + MB), _state(dst=FAR + 2 * MB, src=FAR)], "states 0 and 1"),                       # read while it is written
    ([_state(dst=FAR + 2 * MB, src=FAR), _state(dst=FAR, src=FAR + MB)], "states 0 and 1"),
    ([_state(dst=FAR, src=FAR), _state(dst=FAR + MB, src=FAR + 8191)], "states 0 and 1"),
    ([_state(dst=FAR + i * MB, src=FAR + i * MB) for i in range(40)] + [_state(dst=FAR + 7 * MB + 8191, src=FAR + 99 * MB)], "states 7 and 40"),
    ([_state(dst=FAR, src=FAR, nbytes=256), _state(dst=FAR + 255, src=FAR + 255, nbytes=256)], "states 0 and 1"),  # halves of rows that meet
    ([_state(dst=FAR, src=FAR + 512 * 3)], "dst and src of state 0 overlap"),
    ([_state(), _state(dst=FAR, src=FAR + 99 * MB, ds=1 << 24, dr=1 << 20), _state(dst=AT - 8191, src=FAR + 300 * MB)], "states 0 and 2"),
])
def test_reorder_refuses_states_that_share_memory(states, frag):
    _refused(_reorder(states, back=AT + 32 * MB), frag)


@pytest.mark.parametrize("back", [AT, AT + 8191, AT - 63])
def test_reorder_refuses_back_pointers_in_a_dst(back):
    _refused(_reorder([_state(nbytes=0), _state()], back=back), "backptr_dev lies in state 1")


def test_reorder_refuses_what_it_cannot_tell_apart():
    """Bytes 6 and 9 apart, which never meet, in rows of different strides."""
    a = _state(dst=FAR, src=FAR + 900 * MB, ds=8 * 40968, dr=40968, dg=6, ss=8 * 40968, sr=40968, sg=6, segs=6000, nbytes=1)
    b = _state(dst=FAR + 1, src=FAR + 1900 * MB, ds=8 * 36009, dr=36009, dg=9, ss=8 * 36009, sr=36009, sg=9, segs=4000, nbytes=1)
    _refused(_reorder([a, b], B=64), "states 0 and 1")


# 2 sentences of 4 rows of 100 fp32 logits, 104 apart; everything else lies apart
APART = dict(logits=FAR, rs=104, ss=500, score=AT, flags=AT + 4096, tok=AT + (1 << 13), back=AT + (2 << 13), osc=AT + (3 << 13), ofl=AT + (4 << 13), ws=AT + MB)


@pytest.mark.parametrize("kw,frag", [
    (dict(tok=FAR), "in the logits"), (dict(back=FAR + 500 * 4 + 104 * 4 * 3 + 396), "in the logits"), (dict(osc=FAR - 31), "in the logits"), (dict(ofl=FAR + 400 - 1), "in the logits"),
    (dict(tok=APART["back"]), "arrays of the new beam"), (dict(osc=APART["back"] + 31), "arrays of the new beam"), (dict(ofl=APART["tok"] + 8), "arrays of the new beam"),
    (dict(tok=APART["ws"]), "beam lies in the workspace"), (dict(ofl=APART["ws"] + 64), "beam lies in the workspace"), (dict(osc=APART["ws"] - 31), "beam lies in the workspace"),
    (dict(score=APART["ws"] + 4), "input lies in the workspace"), (dict(flags=APART["ws"] - 7), "input lies in the workspace"), (dict(logits=APART["ws"] - 2000), "input lies in the workspace"),
])
def test_select_refuses_what_shares_memory(kw, frag):
    _refused(_select(**{**APART, **kw}), frag)


# 2 sentences of 3 tokens of 8 query heads (4 of the cache's) of 64 in bf16: 8192, 1024 and 64 elements between them
POOL = _cache(k=AT + 512 * MB, v=AT + 600 * MB)


def _tensor(i, **kw):
    return _heads(data=FAR + i * MB, **kw)


@pytest.mark.parametrize("kw,frag", [
    (dict(cache=_cache(page_stride=0)), "tokens of the cache"), (dict(cache=_cache(token_stride=0)), "tokens of the cache"), (dict(cache=_cache(head_stride=56)), "tokens of the cache"),
    (dict(q_out=_tensor(3, s=0)), "pieces of q_out"), (dict(q_out=_tensor(3, t=0)), "pieces of q_out"), (dict(q_out=_tensor(3, h=56)), "pieces of q_out"),
    (dict(q_out=_heads(data=FAR + 2 * MB + 16)), "overlaps"), (dict(q_out=_tensor(0)), "overlaps"), (dict(q_out=_heads(data=FAR + MB + 16384)), "overlaps"),
    (dict(q_out=_heads(data=FAR + 2 * MB - 2 * 10240 + 128)), "overlaps"),
])
def test_append_refuses_what_shares_memory(kw, frag):
    _refused(_append(**{**dict(cache=POOL, k=_tensor(0), v=_tensor(1), q=_tensor(2), q_out=_tensor(3)), **kw}), frag)


@pytest.mark.parametrize("kw,frag", [
    (dict(out=_tensor(3, s=0)), "pieces of out"), (dict(out=_tensor(3, t=0)), "pieces of out"), (dict(out=_tensor(3, h=56)), "pieces of out"),
    (dict(out=_heads(data=FAR + 2 * MB + 16)), "part of q"), (dict(out=_tensor(2, t=512)), "part of q"), (dict(out=_tensor(9, s=0)), "pieces of out"),
    (dict(lse=FAR + 2 * MB), "out_lse_dev"), (dict(lse=FAR + 3 * MB + 1024 * 2 * 2 + 1020), "out_lse_dev"),
    (dict(ws=FAR + 2 * MB), "workspace"), (dict(ws=FAR + 3 * MB + 256), "workspace"), (dict(lse=FAR + 20 * MB), "workspace"),
])
def test_attend_refuses_what_shares_memory(kw, frag):
    """Of one head of 10000 tokens, which takes a workspace."""
    cache = _cache(k=AT + 512 * MB, v=AT + 600 * MB, max_pages=4096, table_stride=4096)
    a = {**dict(q=_tensor(2), out=_tensor(3), lse=FAR + 4 * MB, ws=FAR + 20 * MB), **kw}
    r = ctypes.byref
    _refused(beam.load().dba_tree_attend(2, 3, 8, r(a["q"]), r(cache), AT, AT, AT, 1, 10000, 0.125, r(a["out"]), a["lse"], a["ws"], 1 << 40, None), frag)
