"""-m "not gpu": calls of the operators whose tensors share memory that is written are refused before the device is touched."""
import pytest

from test_beam_ops_cpu import AT, _refused, _reorder, _select, _state

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
