"""-m "not gpu": what the binding packs for a call is laid out as the structures of include/dba_beam.h."""
import ctypes

import pytest
import torch

from paper_1804_06609_amd import beam, binding


def fields(struct):
    return {name: getattr(struct, name) for name, _ in struct._fields_}


def test_a_cache():
    k, v = (torch.zeros(5, 8, 3, 16, dtype=torch.float16) for _ in range(2))
    table = torch.zeros(2, 7, dtype=torch.int32)[:, :4]
    got = beam._Cache.from_buffer_copy(beam._cache(k, v, table, 2, torch.float16, -1))
    assert fields(got) == dict(k=k.data_ptr(), v=v.data_ptr(), table=table.data_ptr(), table_stride=7, page_stride=384, token_stride=48, head_stride=16,
                               format=binding.DBA_LOGP_F16, n_pages=5, page_size=8, max_pages=4, heads=3, head_dim=16)
    assert len(beam._cache(k, v, table, 2, torch.float16, -1)) == ctypes.sizeof(beam._Cache)


@pytest.mark.parametrize("shape,strides", [((2, 3, 4, 8), (96, 32, 8)), ((1, 3, 4, 8), (0, 32, 8)), ((2, 1, 1, 8), (8, 0, 0))])
def test_heads(shape, strides):
    x = torch.zeros(shape)
    packed = beam._heads("x", x, shape, torch.float32, -1)
    got = beam._Heads.from_buffer_copy(packed)
    assert len(packed) == ctypes.sizeof(beam._Heads) and tuple(fields(got).values()) == (x.data_ptr(),) + strides


def test_states():
    values = list(range(100, 120))
    packed = beam._pack_states(20)(*values)
    assert len(packed) == 2 * ctypes.sizeof(beam._State)
    got = (beam._State * 2).from_buffer_copy(packed)
    assert [list(fields(s).values()) for s in got] == [values[:10], values[10:]]
    assert list(fields(got[0])) == ["dst", "src", "dst_sent", "dst_row", "dst_seg", "src_sent", "src_row", "src_seg", "segs", "seg_bytes"]
