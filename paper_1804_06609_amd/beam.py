"""The operators of include/dba_beam.h on torch tensors: marshalling and device-memory plumbing only.

`select` (the new beam from logits), `reorder` (states follow the back-pointers), `append` (keys and values into a paged
cache, normed and rotated on the way), `attend` (a tree's nodes over that cache), `attend_shared` (the same behind a prefix that the
whole batch has in common), `weigh` (how much attention each cached token has had) and `evict` (those that had the most
stay, in other pages).  All enqueue their work on the current stream of the current device, where their tensors have to be, and return without waiting; workspaces come from torch's allocator on that
stream.  A tensor that was made on another stream is the caller's to wait for, as with any torch operator.
Nothing of the methods runs here, and there is no fallback: without the built library the calls raise.  None has a gradient, and
inputs that require one are refused where torch would record it.
"""
from __future__ import annotations

import ctypes
import functools
import struct
from typing import Optional, Sequence

import torch

from . import binding as _b

_P, _I, _L, _Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t


class _State(ctypes.Structure):
    _fields_ = [("dst", _P), ("src", _P)] + [(f, _L) for f in (
        "dst_sent", "dst_row", "dst_seg", "src_sent", "src_row", "src_seg", "segs", "seg_bytes")]


class _Cache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("table", _P), ("table_stride", _L), ("page_stride", _L), ("token_stride", _L),
                ("head_stride", _L), ("format", _I), ("n_pages", _I), ("page_size", _I), ("max_pages", _I), ("heads", _I), ("head_dim", _I)]


class _Heads(ctypes.Structure):
    _fields_ = [("data", _P), ("sent_stride", _L), ("token_stride", _L), ("head_stride", _L)]


_SIGNATURES = {
    "dba_beam_select_workspace_bytes": (_Z, [_I] * 5),
    "dba_beam_select": (_I, [_I] * 6 + [_P, _I, _L, _L] + [_P] * 6 + [_P, _Z, _P]),
    "dba_beam_reorder": (_I, [_I, _I, _P, _P, _I, _P]),
    "dba_cache_append": (_I, [_I, _I, _P, _P, _P, _I] + [_P] * 6 + [_I, _I, _P]),
    "dba_tree_attend_workspace_bytes": (_Z, [_I, _I, _I, _P, _I]),
    "dba_tree_attend": (_I, [_I, _I, _I] + [_P] * 5 + [_I, _I, ctypes.c_float] + [_P] * 3 + [_Z, _P]),
    "dba_cache_append_normed": (_I, [_I, _I, _P, _P, _P, _I] + [_P] * 6 + [_I, _P, _P, _I, _I, _P]),
    "dba_shared_attend_workspace_bytes": (_Z, [_I, _I, _I, _P, _I, _I, _I]),
    "dba_shared_attend": (_I, [_I, _I, _I, _P, _P, _P, _I, _P, _I, _P, _P, _P, _I, _I, ctypes.c_float] + [_P] * 3 + [_Z, _P]),
    "dba_cache_weigh": (_I, [_I, _I, _I] + [_P] * 6 + [_I, _P, _I, ctypes.c_float, _I, _P, _L, _L, _P, _L, _L, _I, _P, _Z, _P]),
    "dba_cache_weigh_workspace_bytes": (_Z, [_I, _I, _I, _P, _I, _I]),
    "dba_cache_evict_workspace_bytes": (_Z, [_I, _P, _I, _I, _I]),
    "dba_cache_evict": (_I, [_I, _P, _P, _L, _I, _I, _P, _L, _L, _P, _P, _I, _P, _I, _I, _I, _P, _P, _L, _L, _I, _P, _Z, _P]),
}


class _Norms(ctypes.Structure):
    _fields_ = [("q_weight", _P), ("k_weight", _P), ("q_stride", _L), ("k_stride", _L), ("format", _I), ("eps", ctypes.c_float)]


# the same structures as bytes, which are made in half the time
_pack_cache = struct.Struct("@3P4q6i").pack
_pack_heads = struct.Struct("@P3q").pack
_pack_norms = struct.Struct("@2P2qif").pack


@functools.lru_cache(maxsize=256)
def _pack_states(fields: int):
    return struct.Struct(f"@{fields}q").pack


_F32, _I32, _U8, _empty_like, _CONTIGUOUS = torch.float32, torch.int32, torch.uint8, torch.empty_like, torch.contiguous_format
_grad_enabled = torch.is_grad_enabled
_FORMATS = {torch.float32: _b.DBA_LOGP_F32, torch.float16: _b.DBA_LOGP_F16, torch.bfloat16: _b.DBA_LOGP_BF16}

_lib = None


def load() -> ctypes.CDLL:
    """The built library with these operators' signatures; raises if it has not been built."""
    global _lib
    if _lib is None:
        lib = _b.load()
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _fail(text: str):
    raise _b.DbaError(_b.DBA_EINVAL, text)


def _no_gradient():
    """What came out would be cut off from tensors that require a gradient without a word."""
    _fail("this operator has no gradient: call it under torch.no_grad(), or on detached tensors")


def _stream(x: torch.Tensor) -> int:
    if not x.is_cuda:
        _fail("tensors must be on the GPU")
    index = x.get_device()
    if index != torch._C._cuda_getDevice():
        _fail("tensors must be on the current device")
    return torch._C._cuda_getCurrentRawStream(index)       # (torch.cuda.current_stream() takes 2.8 us to say the same)


def _ints(name: str, x: Optional[torch.Tensor], shape, device: int) -> Optional[int]:
    """Address of a dense int32 tensor of this shape (None where it may be left out)."""
    if x is None:
        return None
    if x.dtype is not _I32 or x.shape != shape or x.get_device() != device or not x.is_contiguous():
        _fail(f"{name} must be a contiguous int32 tensor {tuple(shape)} on the device of the others")
    return x.data_ptr()


def _workspace(nbytes: int, like: torch.Tensor):
    """(tensor, address): torch's allocations start on 512 bytes."""
    if not nbytes:
        return None, None
    ws = like.new_empty(nbytes, dtype=_U8)
    return ws, ws.data_ptr()


def select(logits: torch.Tensor, score: torch.Tensor, flags: Optional[torch.Tensor], k_out: int, eos_id: int, pad_id: int,
           out: Optional[Sequence[torch.Tensor]] = None):
    """The new beam from logits [B, k_in, V] (fp32, fp16 or bf16; last axis dense), score [B, k_in] fp32 and flags [B, k_in] uint8 or
    None: (token, backptr, score, flags), each [B, k_out] as dba_step writes them.  `out`: four tensors to write to, apart from each other and from what is read."""
    lib = load()
    if _grad_enabled() and (logits.requires_grad or score.requires_grad):
        _no_gradient()
    shape, fmt = logits.shape, _FORMATS.get(logits.dtype)
    if len(shape) != 3 or fmt is None:
        _fail("logits must be [B, k, V] of fp32, fp16 or bf16 with a dense last axis")
    B, k, V = shape
    sent, row, one = logits.stride()
    if one != 1 and V > 1:
        _fail("logits must be [B, k, V] of fp32, fp16 or bf16 with a dense last axis")
    stream, device, of_rows = _stream(logits), logits.get_device(), (B, k)
    if score.dtype is not _F32 or score.shape != of_rows or not score.is_contiguous() or score.get_device() != device:
        _fail("score must be a contiguous fp32 tensor [B, k] on the device of the logits")
    if flags is not None and (flags.dtype is not _U8 or flags.shape != of_rows or not flags.is_contiguous() or flags.get_device() != device):
        _fail("flags must be a contiguous uint8 tensor [B, k] on the device of the logits")
    if out is None:
        like = score if k_out == k else score.new_empty((B, k_out))
        out = (_empty_like(like, dtype=_I32), _empty_like(like, dtype=_I32), _empty_like(like), _empty_like(like, dtype=_U8))
    else:
        for x, dtype in zip(out, (_I32, _I32, _F32, _U8), strict=True):
            if x.dtype is not dtype or x.shape != (B, k_out) or not x.is_contiguous() or x.get_device() != device:
                _fail("out must be four contiguous tensors [B, k_out]: int32, int32, fp32, uint8")
    nbytes = lib.dba_beam_select_workspace_bytes(B, k, k_out, V, fmt)
    ws, at = _workspace(nbytes, logits)
    _b._check(lib.dba_beam_select(B, k, k_out, V, eos_id, pad_id, logits.data_ptr(), fmt, sent, row,
                                  score.data_ptr(), None if flags is None else flags.data_ptr(), out[0].data_ptr(), out[1].data_ptr(),
                                  out[2].data_ptr(), out[3].data_ptr(), at, nbytes, stream))
    return tuple(out)


@functools.lru_cache(maxsize=1024)
def _pieces(shape, strides, e: int):
    """[B, k, ...] as (sent, row, seg strides in bytes, pieces, bytes of a piece); the axes behind the second fold into two."""
    i, dense = len(shape) - 1, 1                       # dense: elements of a piece so far
    while i > 1 and (strides[i] == dense or shape[i] == 1):
        dense *= shape[i]
        i -= 1
    seg, seg_stride = 1, 0
    while i > 1:
        if shape[i] != 1:
            if seg == 1:
                seg_stride = strides[i]
            elif strides[i] != seg_stride * seg:
                return None
            seg *= shape[i]
        i -= 1
    return strides[0] * e, strides[1] * e, seg_stride * e, seg, dense * e


def reorder(backptr: torch.Tensor, states: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None):
    """Every state [B, k, ...] (any type) follows backptr [B, k] int32: out[b, h] = state[b, backptr[b, h]], rows of a
    back-pointer outside [0, k) cleared.  out None: in place.  Views of the places in use do: behind the
    second axis a state may have one more that is not dense (e.g. [B, k, heads, capacity, width][:, :, :, :t]).  All are moved at the
    same time: what is written lies in no other state, nor in its out.  Returns `out`."""
    lib = load()
    if backptr.dim() != 2:
        _fail("backptr must be [B, k]")
    out = states if out is None else out
    if len(out) != len(states):
        _fail("as many tensors out as states")
    if _grad_enabled():
        for s in states:
            if s.requires_grad:
                _no_gradient()
    B, k = backptr.shape
    stream = _stream(backptr)
    device = backptr.get_device()
    back = _ints("backptr", backptr, backptr.shape, device)
    table = []                                         # the fields of dba_state, one state after another
    rows = B * k or 1
    for s, d in zip(states, out):
        shape = s.shape
        if d.shape != shape or len(shape) < 2 or shape[0] != B or shape[1] != k or s.dtype is not d.dtype or s.get_device() != device or d.get_device() != device:
            _fail("states and out must be [B, k, ...] tensors alike in shape and type, on the device of backptr")
        if s.is_contiguous() and d.is_contiguous():
            row = s.nbytes // rows
            sent = row * k
            table += (d.data_ptr(), s.data_ptr(), sent, row, 0, sent, row, 0, 1, row)
            continue
        a, c = _pieces(shape, s.stride(), s.element_size()), _pieces(shape, d.stride(), d.element_size())
        if a is None or c is None:
            _fail("a state's axes behind the second must fold into pieces of one stride")
        if a[3:] != c[3:]:                             # one side is more finely cut: the smaller piece serves both
            piece = min(a[4], c[4])
            if max(a[4], c[4]) % piece or (a[3] > 1 and c[3] > 1):
                _fail("the axes of a state and its out must fold alike")
            a, c = ((x[0], x[1], piece if x[4] > piece else x[2], x[3] * x[4] // piece, piece) for x in (a, c))
        table += (d.data_ptr(), s.data_ptr(), *c[:3], *a)
    _b._check(lib.dba_beam_reorder(B, k, back, _pack_states(len(table))(*table), len(states), stream))
    return out


def _cache(k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, B: int, dtype, device: int) -> bytes:
    shape = k_pages.shape
    if len(shape) != 4 or v_pages.shape != shape:
        _fail("k_pages and v_pages must be [pages, page_size, heads, head_dim]")
    n_pages, page, heads, D = shape
    s, r = k_pages.stride(), v_pages.stride()
    if s != r or page == 1 or heads == 1 or n_pages == 1:  # the stride of an axis of one is never used; torch gives it any value
        s, r = ([st if size > 1 else 0 for st, size in zip(x, shape)] for x in (s, r))
    if s != r or (D > 1 and s[3] != 1):
        _fail("k_pages and v_pages must be laid out alike, with a dense last axis")
    if k_pages.dtype is not dtype or v_pages.dtype is not dtype or dtype not in _FORMATS:
        _fail("keys, values, queries and pages must be of one type: fp32, fp16 or bf16")
    pages_of = table.shape
    if len(pages_of) != 2 or table.dtype is not torch.int32 or pages_of[0] != B:
        _fail("table must be an int32 tensor [B, max_pages] with a dense last axis")
    row, one = table.stride()
    if one != 1:
        _fail("table must be an int32 tensor [B, max_pages] with a dense last axis")
    if k_pages.get_device() != device or v_pages.get_device() != device or table.get_device() != device:
        _fail("tensors must be on one device")
    return _pack_cache(k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), row, s[0], s[1], s[2],
                       _FORMATS[dtype], n_pages, page, pages_of[1], heads, D)


def _heads(name: str, x: torch.Tensor, shape, dtype, device: int) -> bytes:
    if x.shape != shape:
        _fail(f"{name} must be [B, n, heads, head_dim], here {tuple(shape)}")
    sent, token, head, one = x.stride()
    B, n, heads, D = shape
    if x.dtype is not dtype or x.get_device() != device or (one != 1 and D > 1):
        _fail(f"{name} must be of the type and on the device of the others, with a dense last axis")
    return _pack_heads(x.data_ptr(), sent if B > 1 else 0, token if n > 1 else 0, head if heads > 1 else 0)


def append(k: torch.Tensor, v: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, first: torch.Tensor,
           count: Optional[torch.Tensor] = None, *, position: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None,
           interleaved: bool = False, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, axis: Optional[torch.Tensor] = None,
           eps: Optional[float] = None, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """k, v [B, n, heads, head_dim] become tokens first[b] .. of the cache (count[b] of them, or n), k rotated by its position ([B, n]
    int32, or first[b] + i) and inv_freq (fp32; None: no rotation).  q [B, n, q_heads, head_dim] is rotated alike into q_out (a new
    tensor if None; q itself is allowed), which is returned.

    With axis ([rot_dim / 2] int32) positions are [B, n, axes] and pair j goes by axis[j] of them.  With eps, queries and keys are
    normed by head before they are rotated: x / sqrt(mean x^2 + eps), times q_weight or k_weight where there is one ([head_dim], or one
    for each head [heads, head_dim]; of the queries' type or fp32)."""
    lib = load()
    if axis is not None or eps is not None or q_weight is not None or k_weight is not None:
        return _append_normed(lib, k, v, k_pages, v_pages, table, first, count, position, inv_freq, interleaved, q, q_out, axis, eps, q_weight, k_weight)
    if _grad_enabled() and (k.requires_grad or v.requires_grad or (q is not None and q.requires_grad) or (inv_freq is not None and inv_freq.requires_grad)):
        _no_gradient()
    stream = _stream(k)
    shape, dtype, device = k.shape, k.dtype, k.get_device()
    if len(shape) != 4:
        _fail("k must be [B, n, heads, head_dim]")
    B, n, heads, D = shape
    cache = _cache(k_pages, v_pages, table, B, dtype, device)
    if k_pages.shape[2:] != (heads, D):
        _fail("k has other heads than the cache")
    qh = oh = None
    q_heads = 0
    if q is not None:
        if q.dim() != 4:
            _fail("q must be [B, n, q_heads, head_dim]")
        q_heads = q.shape[2]
        if q_out is None:
            q_out = _empty_like(q, memory_format=_CONTIGUOUS)
        qh, oh = _heads("q", q, (B, n, q_heads, D), dtype, device), _heads("q_out", q_out, (B, n, q_heads, D), dtype, device)
    rot, freq = 0, None
    if inv_freq is not None:
        if inv_freq.dtype is not torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous() or inv_freq.get_device() != device:
            _fail("inv_freq must be a contiguous fp32 tensor [rot_dim / 2]")
        rot, freq = 2 * inv_freq.shape[0], inv_freq.data_ptr()
    _b._check(lib.dba_cache_append(B, n, cache, _heads("k", k, shape, dtype, device), _heads("v", v, shape, dtype, device), q_heads, qh, oh,
                                   _ints("first", first, (B,), device), _ints("count", count, (B,), device),
                                   _ints("position", position, (B, n), device), freq, rot, interleaved, stream))
    return q_out


def _weights(name: str, w: Optional[torch.Tensor], heads: int, D: int, device: int):
    """(address, elements between heads) of the weights of norms."""
    if w is None:
        return 0, 0
    if w.shape != (D,) and w.shape != (heads, D) or not w.is_contiguous() or w.get_device() != device:
        _fail(f"{name} must be contiguous, [head_dim] or [heads, head_dim], on the device of the others")
    return w.data_ptr(), D if w.dim() == 2 and heads > 1 else 0


def _append_normed(lib, k, v, k_pages, v_pages, table, first, count, position, inv_freq, interleaved, q, q_out, axis, eps, q_weight, k_weight):
    """`append` where there are norms, or positions of several axes."""
    if _grad_enabled() and any(x is not None and x.requires_grad for x in (k, v, q, inv_freq, q_weight, k_weight)):
        _no_gradient()
    stream = _stream(k)
    shape, dtype, device = k.shape, k.dtype, k.get_device()
    if len(shape) != 4:
        _fail("k must be [B, n, heads, head_dim]")
    B, n, heads, D = shape
    cache = _cache(k_pages, v_pages, table, B, dtype, device)
    if k_pages.shape[2:] != (heads, D):
        _fail("k has other heads than the cache")
    qh = oh = None
    q_heads = 0
    if q is not None:
        if q.dim() != 4:
            _fail("q must be [B, n, q_heads, head_dim]")
        q_heads = q.shape[2]
        if q_out is None:
            q_out = _empty_like(q, memory_format=_CONTIGUOUS)
        qh, oh = _heads("q", q, (B, n, q_heads, D), dtype, device), _heads("q_out", q_out, (B, n, q_heads, D), dtype, device)
    rot, freq, norms, axes = 0, None, None, 1
    if inv_freq is not None:
        if inv_freq.dtype is not _F32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous() or inv_freq.get_device() != device:
            _fail("inv_freq must be a contiguous fp32 tensor [rot_dim / 2]")
        rot, freq = 2 * inv_freq.shape[0], inv_freq.data_ptr()
    if axis is not None:
        if position is None or position.dim() != 3 or inv_freq is None:
            _fail("axis goes with positions [B, n, axes] and inv_freq")
        axes = position.shape[2]
    if eps is not None:
        kinds = {w.dtype for w in (q_weight, k_weight) if w is not None} or {dtype}
        kind = kinds.pop()
        if kinds or (kind is not dtype and kind is not _F32):
            _fail("weights of norms must be of one type, the queries' or fp32")
        a, sa = _weights("q_weight", q_weight, q_heads, D, device)
        c, sc = _weights("k_weight", k_weight, heads, D, device)
        norms = _pack_norms(a, c, sa, sc, _FORMATS[kind], eps)
    elif q_weight is not None or k_weight is not None:
        _fail("weights of norms go with eps")
    _b._check(lib.dba_cache_append_normed(B, n, cache, _heads("k", k, shape, dtype, device), _heads("v", v, shape, dtype, device), q_heads, qh, oh, norms,
                                          _ints("first", first, (B,), device), _ints("count", count, (B,), device),
                                          _ints("position", position, (B, n) if axis is None else (B, n, axes), device), axes,
                                          _ints("axis", axis, (rot // 2,), device), freq, rot, interleaved, stream))
    return q_out


def _mask(mask: Optional[torch.Tensor], B: int, n: int, device: int):
    """(words of a node, address, whether there is a mask without a bit)."""
    if mask is None:
        return 0, None, False
    if mask.dtype is not torch.int64 or mask.dim() != 3 or mask.shape[:2] != (B, n) or not mask.is_contiguous() or mask.get_device() != device:
        _fail("mask must be a contiguous int64 tensor [B, n, words] on the device of the others")
    words = mask.shape[2]
    return words, mask.data_ptr() if words else None, not words


def attend(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, prefix: torch.Tensor,
           tree: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, *, scale: Optional[float] = None,
           max_len: Optional[int] = None, out: Optional[torch.Tensor] = None, return_lse: bool = False):
    """q [B, n, q_heads, head_dim] over the cache: node i of sentence b sees its prefix[b] first tokens and, of the tree[b] behind
    them, those whose bit is set in mask [B, n, words] (int64, 64 tokens a word, lowest bit first); without a mask the n nodes are
    the last n tokens of a chain.  scale: head_dim ** -0.5 if None.  max_len: no sentence has more tokens (the table's capacity
    if None; a close bound makes a better launch).  Returns out, or (out, lse [B, n, q_heads] fp32)."""
    lib = load()
    if _grad_enabled() and (q.requires_grad or k_pages.requires_grad or v_pages.requires_grad):
        _no_gradient()
    stream = _stream(q)
    shape, dtype, device = q.shape, q.dtype, q.get_device()
    if len(shape) != 4:
        _fail("q must be [B, n, q_heads, head_dim]")
    B, n, heads, D = shape
    cache = _cache(k_pages, v_pages, table, B, dtype, device)
    if k_pages.shape[3] != D:
        _fail("q has another head_dim than the cache")
    if out is None:
        out = _empty_like(q, memory_format=_CONTIGUOUS)
    words, bits = 0, None
    if mask is not None:
        if mask.dtype is not torch.int64 or mask.dim() != 3 or mask.shape[:2] != (B, n) or not mask.is_contiguous() or mask.get_device() != device:
            _fail("mask must be a contiguous int64 tensor [B, n, words] on the device of the others")
        words = mask.shape[2]
        if words:
            bits = mask.data_ptr()
        else:                                              # a mask without a bit: nothing of the tree is seen
            tree = None
    lse = q.new_empty((B, n, heads), dtype=torch.float32) if return_lse else None
    if max_len is None:
        max_len = min(table.shape[1] * k_pages.shape[1], 2**31 - 1024)
    nbytes = lib.dba_tree_attend_workspace_bytes(B, n, heads, cache, max_len)
    ws, at = _workspace(nbytes, q)
    _b._check(lib.dba_tree_attend(B, n, heads, _heads("q", q, shape, dtype, device), cache, _ints("prefix", prefix, (B,), device),
                                  _ints("tree", tree, (B,), device), bits, words, max_len, D ** -0.5 if scale is None else scale,
                                  _heads("out", out, shape, dtype, device), lse.data_ptr() if return_lse else None, at, nbytes, stream))
    return (out, lse) if return_lse else out


def attend_shared(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, shared: torch.Tensor, shared_len: torch.Tensor, table: torch.Tensor,
                  prefix: torch.Tensor, tree: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, *, scale: Optional[float] = None,
                  max_shared: Optional[int] = None, max_len: Optional[int] = None, out: Optional[torch.Tensor] = None, return_lse: bool = False):
    """`attend` of sentences that have their first tokens in common: every node sees the shared_len ([1] int32) first tokens of the pages
    `shared` ([pages] int32, of the same pools), read once for the whole batch, and what `attend` lets it see of its sentence's own. max_shared:
    there are no more common tokens (the pages' capacity if None).  All else is as for `attend`; the normaliser is that of both together."""
    lib = load()
    if _grad_enabled() and (q.requires_grad or k_pages.requires_grad or v_pages.requires_grad):
        _no_gradient()
    stream = _stream(q)
    shape, dtype, device = q.shape, q.dtype, q.get_device()
    if len(shape) != 4:
        _fail("q must be [B, n, q_heads, head_dim]")
    B, n, heads, D = shape
    cache = _cache(k_pages, v_pages, table, B, dtype, device)
    if k_pages.shape[3] != D:
        _fail("q has another head_dim than the cache")
    if shared.dim() != 1:
        _fail("shared must be [pages]")
    if out is None:
        out = _empty_like(q, memory_format=_CONTIGUOUS)
    words, bits, blind = _mask(mask, B, n, device)
    if blind:                                              # nothing of the tree is seen
        tree = None
    lse = q.new_empty((B, n, heads), dtype=_F32) if return_lse else None
    page, pages = k_pages.shape[1], shared.shape[0]
    if max_len is None:
        max_len = min(table.shape[1] * page, 2**31 - 1024)
    if max_shared is None:
        max_shared = min(pages * page, 2**31 - 1024)
    nbytes = lib.dba_shared_attend_workspace_bytes(B, n, heads, cache, pages, max_shared, max_len)
    ws, at = _workspace(nbytes, q)
    _b._check(lib.dba_shared_attend(B, n, heads, _heads("q", q, shape, dtype, device), cache, _ints("shared", shared, shared.shape, device), pages,
                                    _ints("shared_len", shared_len, (1,), device), max_shared, _ints("prefix", prefix, (B,), device),
                                    _ints("tree", tree, (B,), device), bits, words, max_len, D ** -0.5 if scale is None else scale,
                                    _heads("out", out, shape, dtype, device), lse.data_ptr() if return_lse else None, at, nbytes, stream))
    return (out, lse) if return_lse else out


def _scores(name: str, x: torch.Tensor, shape, device: int):
    """(address, strides of sentences and heads) of fp32 scores [B, 1 or heads, width]."""
    if x.dtype is not _F32 or x.shape != shape or x.get_device() != device:
        _fail(f"{name} must be an fp32 tensor {tuple(shape)} on the device of the others")
    sent, head, one = x.stride()
    if one != 1 and shape[2] > 1:
        _fail(f"{name} must have a dense last axis")
    return x.data_ptr(), sent if shape[0] > 1 else 0, head if shape[1] > 1 else 0


def weigh(score: torch.Tensor, q: torch.Tensor, lse: torch.Tensor, k_pages: torch.Tensor, table: torch.Tensor, prefix: torch.Tensor,
          tree: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, *, count: Optional[torch.Tensor] = None,
          scale: Optional[float] = None, max_len: Optional[int] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """score [B, heads, width] (a score for each head of the cache) or [B, 1, width] (one for all), fp32, plus the attention weight that each cached
    token has from q [B, n, q_heads, head_dim] with normalisers lse [B, n, q_heads], as `attend` or `attend_shared` returned them, of nodes that
    see it; nodes from count[b] on do not count, nor does a head whose lse is not finite.  In place, or into `out`, which is returned."""
    lib = load()
    if _grad_enabled() and (score.requires_grad or q.requires_grad or lse.requires_grad or k_pages.requires_grad):
        _no_gradient()
    stream = _stream(q)
    shape, dtype, device = q.shape, q.dtype, q.get_device()
    if len(shape) != 4:
        _fail("q must be [B, n, q_heads, head_dim]")
    B, n, heads, D = shape
    cache = _cache(k_pages, k_pages, table, B, dtype, device)
    kv_heads = k_pages.shape[2]
    if k_pages.shape[3] != D:
        _fail("q has another head_dim than the cache")
    if lse.dtype is not _F32 or lse.shape != (B, n, heads) or not lse.is_contiguous() or lse.get_device() != device:
        _fail("lse must be a contiguous fp32 tensor [B, n, q_heads] on the device of the others")
    if score.dim() != 3 or score.shape[1] not in (1, kv_heads):
        _fail("score must be [B, heads of the cache, width] or [B, 1, width]")
    rows = (B, score.shape[1], score.shape[2])
    out = score if out is None else out
    words, bits, blind = _mask(mask, B, n, device)
    if blind:
        tree = None
    if max_len is None:
        max_len = min(table.shape[1] * k_pages.shape[1], rows[2])
    by_head = rows[1] == kv_heads
    nbytes = lib.dba_cache_weigh_workspace_bytes(B, n, heads, cache, by_head, max_len)
    ws, at = _workspace(nbytes, q)
    _b._check(lib.dba_cache_weigh(B, n, heads, _heads("q", q, shape, dtype, device), lse.data_ptr(), cache, _ints("prefix", prefix, (B,), device),
                                  _ints("tree", tree, (B,), device), bits, words, _ints("count", count, (B,), device), max_len,
                                  D ** -0.5 if scale is None else scale, by_head, *_scores("score", score, rows, device),
                                  *_scores("out", out, rows, device), rows[2], at, nbytes, stream))
    return out


def evict(score: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, new_table: torch.Tensor, prefix: torch.Tensor,
          tree: Optional[torch.Tensor] = None, *, keep: int, budget: Optional[torch.Tensor] = None, sinks: int = 0, recent: int = 0,
          max_len: Optional[int] = None, new_score: Optional[torch.Tensor] = None):
    """Of the prefix[b] first tokens of each sentence's cache min(keep, budget[b]) move into the pages of new_table ([B, pages] int32, other pages of the
    same pools), and the tree[b] ones behind them: the `sinks` first and the `recent` last ones before all others, then those of the greatest
    score ([B, heads, width]: each head of the cache chooses its own, or [B, 1, width]), all in their order.  Returns the new prefix [B] int32 and
    the scores of the tokens at their new places, 0 behind them (new_score, or a new tensor like score)."""
    lib = load()
    if _grad_enabled() and (score.requires_grad or k_pages.requires_grad or v_pages.requires_grad):
        _no_gradient()
    stream = _stream(score)
    device = score.get_device()
    if score.dim() != 3 or k_pages.dim() != 4 or score.shape[1] not in (1, k_pages.shape[2]):
        _fail("score must be [B, heads of the cache, width] or [B, 1, width]")
    rows = B, heads, width = tuple(score.shape)
    cache = _cache(k_pages, v_pages, table, B, k_pages.dtype, device)
    if new_table.dtype is not _I32 or new_table.dim() != 2 or new_table.shape[0] != B or new_table.stride(1) != 1 or new_table.get_device() != device:
        _fail("new_table must be an int32 tensor [B, pages] with a dense last axis, on the device of the others")
    if new_score is None:
        new_score = _empty_like(score, memory_format=_CONTIGUOUS)
    new_prefix = prefix.new_empty((B,))
    by_head = heads == k_pages.shape[2]
    keep, sinks, recent = (min(x, 2**31 - 1) for x in (keep, sinks, recent))       # (more than there are tokens)
    if max_len is None:
        max_len = min(table.shape[1] * k_pages.shape[1], width)
    nbytes = lib.dba_cache_evict_workspace_bytes(B, cache, by_head, keep, max_len)
    ws, at = _workspace(nbytes, score)
    _b._check(lib.dba_cache_evict(B, cache, new_table.data_ptr(), new_table.stride(0) if B > 1 else new_table.shape[1], new_table.shape[1], by_head,
                                  *_scores("score", score, rows, device), _ints("prefix", prefix, (B,), device), _ints("tree", tree, (B,), device), keep,
                                  _ints("budget", budget, (B,), device), sinks, recent, max_len, new_prefix.data_ptr(),
                                  *_scores("new_score", new_score, rows, device), width, at, nbytes, stream))
    return new_prefix, new_score
