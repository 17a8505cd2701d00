"""-m "not gpu": the operators of include/dba_beam.h - exports, refusals (which come before the device is touched), the cache's
address arithmetic on the host."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_1804_06609_amd as dba
from paper_1804_06609_amd import beam, binding

HERE = os.path.dirname(os.path.abspath(__file__))
AT = 1 << 20               # an aligned fake device address


def test_header_library_and_binding_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(os.path.dirname(HERE), "include", "dba_beam.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"DBA_API\s+[\w\s\*]+?\b(dba_\w+)\s*\(", text)))
    assert names == sorted(beam._SIGNATURES)
    lib = ctypes.CDLL(binding.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)


@pytest.fixture(scope="module")
def header_from_c(tmp_path_factory):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    d = tmp_path_factory.mktemp("c")
    (d / "x.c").write_text('#include "dba_beam.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu\\n", sizeof(dba_state), '
                           'sizeof(dba_cache), sizeof(dba_heads)); return 0; }\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(os.path.dirname(HERE), "include"), str(d / "x.c"), "-o", str(d / "x")], check=True)
    return subprocess.run([str(d / "x")], capture_output=True, text=True, check=True).stdout


def test_structs_are_laid_out_as_in_c(header_from_c):
    assert header_from_c.split() == [str(ctypes.sizeof(t)) for t in (beam._State, beam._Cache, beam._Heads)]


def _refused(rc, frag, code=dba.DBA_EINVAL):
    assert rc == code
    assert frag in binding.dba_last_error(None)


# ---- selection -------------------------------------------------------------------------------------------------------
def _select(B=2, k_in=4, k_out=4, V=100, eos=2, pad=0, logits=AT, fmt=0, ss=400, rs=100, score=AT, flags=AT, tok=AT, back=AT, osc=AT,
            ofl=AT, ws=AT, nbytes=1 << 30):
    return beam.load().dba_beam_select(B, k_in, k_out, V, eos, pad, logits, fmt, ss, rs, score, flags, tok, back, osc, ofl, ws, nbytes, None)


@pytest.mark.parametrize("kw,frag", [
    (dict(B=0), "B"), (dict(B=65536), "B"), (dict(k_in=0), "k_in"), (dict(k_in=65), "k_in"), (dict(k_out=0), "k_out"), (dict(k_out=65), "k_out"),
    (dict(V=0), "V"), (dict(V=(1 << 24) + 1, rs=1 << 25), "V"), (dict(fmt=3), "format"), (dict(fmt=-1), "format"),
    (dict(eos=100), "eos_id"), (dict(eos=-2), "eos_id"), (dict(pad=-1), "eos_id"), (dict(pad=100), "eos_id"), (dict(eos=0), "eos_id"),
    (dict(logits=None), "NULL"), (dict(score=None), "NULL"), (dict(tok=None), "NULL"), (dict(back=None), "NULL"), (dict(osc=None), "NULL"),
    (dict(ofl=None), "NULL"), (dict(logits=AT + 2), "aligned"), (dict(fmt=1, logits=AT + 1), "aligned"), (dict(rs=99), "row_stride"),
    (dict(ss=-1), "sent_stride"), (dict(ws=None), "256"), (dict(ws=AT + 128), "256"),
])
def test_select_refuses(kw, frag):
    _refused(_select(**kw), frag)


@pytest.mark.parametrize("kw", [dict(osc=AT), dict(tok=AT + 28), dict(back=AT - 28), dict(ofl=AT + 4099), dict(ofl=AT + 31)])
def test_select_refuses_a_new_beam_in_the_old_one(kw):
    """2 x 4 scores from AT, flags 4096 behind; everything else lies apart."""
    apart = dict(tok=AT + (1 << 13), back=AT + (2 << 13), osc=AT + (3 << 13), ofl=AT + (4 << 13), score=AT, flags=AT + 4096, logits=AT + (5 << 13), ws=AT + (6 << 13))
    _refused(_select(**{**apart, **kw}), "old one")


def test_select_workspace():
    size = beam.load().dba_beam_select_workspace_bytes
    assert 0 < size(1, 5, 5, 1000, 0) < 1 << 20
    assert size(65535, 64, 64, 1 << 24, 0) > 1 << 32
    for bad in [(0, 1, 1, 10, 0), (1, 0, 1, 10, 0), (1, 1, 65, 10, 0), (1, 1, 1, 0, 0), (1, 1, 1, 10, 7)]:
        assert size(*bad) == 0
    need = size(2, 4, 4, 100, 0)
    _refused(_select(nbytes=need - 1), "workspace", dba.DBA_ENOMEM)


# ---- reordering ------------------------------------------------------------------------------------------------------
def _state(dst=AT, src=AT + (1 << 16), ds=4096, dr=512, dg=0, ss=4096, sr=512, sg=0, segs=1, nbytes=512):
    return beam._State(dst, src, ds, dr, dg, ss, sr, sg, segs, nbytes)


def _reorder(states, B=2, k=8, back=AT, n=None):
    table = (beam._State * max(1, len(states)))(*states)
    return beam.load().dba_beam_reorder(B, k, back, table, len(states) if n is None else n, None)


@pytest.mark.parametrize("kw,frag", [
    (dict(B=0), "B"), (dict(B=65536), "B"), (dict(k=0), "k"), (dict(k=65), "k"), (dict(n=-1), "n_states"), (dict(back=None), "NULL"),
])
def test_reorder_refuses(kw, frag):
    _refused(_reorder([_state()], **kw), frag)


@pytest.mark.parametrize("kw,frag", [
    (dict(dst=None), "NULL"), (dict(src=None), "NULL"), (dict(segs=-1), "negative size"), (dict(nbytes=-1), "negative size"),
    (dict(dr=511), "overlap"), (dict(ds=4095), "overlap"), (dict(dr=0), "overlap"), (dict(ds=-4096), "overlap"), (dict(segs=2, dg=256, sg=512), "overlap"),
    (dict(sr=-512), "negative stride"), (dict(src=AT, sr=1024, ss=8192), "two sets of strides"), (dict(src=AT + 8191), "overlap"),
    (dict(src=AT - 8191), "overlap"), (dict(nbytes=(1 << 31) + 16, dr=1 << 32, ds=1 << 36, src=1 << 50), "2 GB"),
])
def test_reorder_refuses_a_state(kw, frag):
    _refused(_reorder([_state(nbytes=16), _state(**kw)]), frag)      # the good one before it is not launched


def test_reorder_of_nothing_is_no_launch():
    assert _reorder([]) == dba.DBA_OK
    assert _reorder([_state(nbytes=0, dst=None), _state(segs=0, src=None)]) == dba.DBA_OK


# ---- cache and attention ----------------------------------------------------------------------------------------------
def _cache(k=AT, v=AT, table=AT, table_stride=8, page_stride=16 * 4 * 64, token_stride=4 * 64, head_stride=64, fmt=2, n_pages=100, page=16,
           max_pages=8, heads=4, D=64):
    return beam._Cache(k, v, table, table_stride, page_stride, token_stride, head_stride, fmt, n_pages, page, max_pages, heads, D)


def _heads(data=AT, s=8192, t=1024, h=64):
    return beam._Heads(data, s, t, h)


BAD_CACHES = [
    (dict(fmt=3), "format"), (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(table=None), "NULL"), (dict(heads=0), "heads"),
    (dict(D=0), "head_dim"), (dict(D=12), "head_dim"), (dict(D=264), "head_dim"), (dict(page=0), "page_size"), (dict(page=24), "page_size"),
    (dict(page=1 << 17), "page_size"), (dict(n_pages=0), "n_pages"), (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 27, table_stride=1 << 27), "2^31"),
    (dict(table_stride=7), "table_stride"), (dict(k=AT + 8), "16 bytes"), (dict(v=AT + 2), "16 bytes"), (dict(page_stride=100), "16 bytes"),
    (dict(token_stride=4), "16 bytes"), (dict(head_stride=4), "16 bytes"), (dict(token_stride=-256), "16 bytes"),
]


def _append(cache=None, k=None, v=None, q=None, q_out=None, q_heads=8, B=2, n=3, first=AT, inv=AT, rot=64):
    r = ctypes.byref
    return beam.load().dba_cache_append(B, n, r(cache or _cache()), r(k or _heads()), r(v or _heads()), q_heads, r(q) if q else None,
                                        r(q_out) if q_out else None, first, None, None, inv, rot, 0, None)


@pytest.mark.parametrize("kw,frag", BAD_CACHES)
def test_append_refuses_a_cache(kw, frag):
    _refused(_append(_cache(**kw)), frag)


@pytest.mark.parametrize("kw,frag", [
    (dict(B=0), "B"), (dict(n=0), "n"), (dict(n=(1 << 22) + 1), "n"), (dict(first=None), "first"), (dict(inv=None), "inv_freq"), (dict(rot=8), "rot_dim"),
    (dict(rot=80), "rot_dim"), (dict(rot=-16), "rot_dim"), (dict(k=_heads(data=None)), "NULL"), (dict(v=_heads(t=4)), "16 bytes"),
    (dict(q=_heads()), "together"), (dict(q_out=_heads()), "together"), (dict(q=_heads(), q_out=_heads(), q_heads=0), "q_heads"),
    (dict(q=_heads(), q_out=_heads(t=2048)), "two sets"), (dict(q=_heads(), q_out=_heads(data=AT + 4)), "16 bytes"),
])
def test_append_refuses(kw, frag):
    _refused(_append(**kw), frag)


def _attend(cache=None, q=None, out=None, q_heads=8, B=2, n=3, prefix=AT, tree=AT, mask=AT, words=1, max_len=128, scale=0.125, ws=AT, nbytes=1 << 40):
    r = ctypes.byref
    return beam.load().dba_tree_attend(B, n, q_heads, r(q or _heads()), r(cache or _cache()), prefix, tree, mask, words, max_len, scale,
                                       r(out or _heads()), None, ws, nbytes, None)


@pytest.mark.parametrize("kw,frag", BAD_CACHES)
def test_attend_refuses_a_cache(kw, frag):
    _refused(_attend(_cache(**kw)), frag)


@pytest.mark.parametrize("kw,frag", [
    (dict(B=0), "B"), (dict(B=65536), "B"), (dict(n=0), "n"), (dict(n=1 << 21), "n"), (dict(q_heads=6), "multiple"), (dict(q_heads=0), "q_heads"),
    (dict(prefix=None), "prefix"), (dict(tree=None), "mask"), (dict(words=-1), "mask"), (dict(max_len=0), "max_len"), (dict(max_len=129), "max_len"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(q=_heads(data=None)), "NULL"), (dict(out=_heads(data=AT + 8)), "16 bytes"),
])
def test_attend_refuses(kw, frag):
    _refused(_attend(**kw), frag)


def test_attend_refuses_what_positions_or_the_grid_have_no_room_for():
    long = _cache(page=1, max_pages=2**31 - 1, table_stride=2**31 - 1, n_pages=2**31 - 1)
    _refused(_attend(long, max_len=2**31 - 1023), "2^31 - 1024")
    assert beam.load().dba_tree_attend_workspace_bytes(1, 1, 4, ctypes.byref(long), 2**31 - 1023) == 0
    assert beam.load().dba_tree_attend_workspace_bytes(1, 1, 4, ctypes.byref(long), 2**31 - 1024) > 0
    _refused(_attend(q_heads=8, B=65535, n=1 << 15), "2^28")


def test_tensors_have_to_be_on_the_gpu():
    with pytest.raises(dba.DbaError, match="GPU"):
        beam.select(torch.zeros(1, 2, 8), torch.zeros(1, 2), None, 2, 2, 0)
    with pytest.raises(dba.DbaError, match="GPU"):
        beam.reorder(torch.zeros(1, 2, dtype=torch.int32), [])


@pytest.mark.parametrize("make,want", [
    (lambda: torch.zeros(2, 3), (12, 4, 0, 1, 4)),
    (lambda: torch.zeros(2, 3, 5, 7), (420, 140, 0, 1, 140)),
    (lambda: torch.zeros(2, 3, 4, 10, 8)[:, :, :, :6], (3840, 1280, 320, 4, 192)),
    (lambda: torch.zeros(2, 3, 2, 4, 10, 8)[:, :, :, :, :6], (7680, 2560, 320, 8, 192)),
    (lambda: torch.zeros(2, 3, 4, 10, 8, dtype=torch.int16)[..., :5], (1920, 640, 16, 40, 10)),
    (lambda: torch.zeros(2, 3, 4, 5, 10, 8)[:, :, :, :2, :6], None),
])
def test_pieces_of_a_state(make, want):
    x = make()
    assert beam._pieces(x.shape, x.stride(), x.element_size()) == want


# ---- the cache's addresses ---------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("paged") / "paged_driver")
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover", os.path.join(HERE, "paged_driver.cpp"), "-o", exe],
                   check=True, timeout=300)
    return lambda *a: [int(x) for x in subprocess.run([exe, *map(str, a)], capture_output=True, text=True, check=True).stdout.split()]


def test_offset_of_a_token(driver):
    table = [3, 9, -1, 10, 0, 2**31 - 1, -2**31, 1]            # two sentences of four pages of 8 tokens, ten pages in the pool
    for b in range(2):
        for t in range(-3, 40):
            page = table[4 * b + t // 8] if 0 <= t < 32 else -1
            want = page * 1000 + t % 8 * 100 if 0 <= page < 10 else -1
            assert driver("offset", 10, 3, 4, 1000, 100, 4, b, t, *table) == [want]


def test_offset_beyond_32_bits(driver):
    assert driver("offset", 1 << 20, 4, 2, 1 << 20, 1 << 16, 2, 0, 17, 5, (1 << 20) - 1) == [((1 << 20) - 1 << 20) + (1 << 16)]
    assert driver("offset", 4, 16, 3, 1 << 40, 1 << 20, 3, 0, (1 << 17) + 65535, 1, 2, 3) == [(3 << 40) + (65535 << 20)]


@pytest.mark.parametrize("prefix,tree,limit,want", [
    (5, 3, 100, [5, 8]), (0, 0, 100, [0, 0]), (-4, 3, 100, [0, 3]), (5, -3, 100, [5, 5]), (99, 3, 100, [99, 100]), (200, 3, 100, [100, 100]),
    (2**31 - 1, 2**31 - 1, 100, [100, 100]), (-2**31, -2**31, 1, [0, 0]),
])
def test_span(driver, prefix, tree, limit, want):
    assert driver("span", prefix, tree, limit) == want
