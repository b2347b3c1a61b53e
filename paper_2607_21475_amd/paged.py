"""The paged cache in front of the eviction: binding and helpers (no method arithmetic).

    ebd_rope            rotary positions of query or key rows
    ebd_append_paged    new tokens into their sequences' pages, keys rotated on the way, queries too
    ebd_attend_paged    attention of a chunk of new tokens, or of a decode step, over the pages
    ebd_gather_paged    the pages read out as units, which ebd_scores and ebd_evict take
    ebd_norm_rope       norms of heads and rotary positions in one pass; ebd_norm_rope_backward: their gradients
    ebd_append_norm     ebd_append_paged for models that normalise queries and keys for each head
    ebd_attend_tree     attention of trees of drafted tokens over the pages
    ebd_keep_rows       the rows of a tree's accepted path moved together
    ebd_plan_step       page tables, slots, positions and tree masks of a step, from the new token counts

Each call takes a parameter struct (`rope_params`, `append_paged_params`, ...) that a program makes once
per plan and keeps: it holds the tables' addresses and the rows' strides.  A struct keeps the tensors
whose addresses it holds alive, and the tensors of a call must have the shapes and strides it was made for.
`PagedCache` holds a pool and makes the structs and outputs of each call; `rope_frequencies` gives the
frequencies of the usual rotary positions.
"""
from __future__ import annotations

import builtins
import ctypes
import math
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import EBD_WS_ATTEND_PAGED, EBD_WS_ATTEND_TREE, EBD_WS_PLAN_STEP, HEAD_DIM, _check, _lib, _ptr, ebd_workspace_size, workspace

EBD_ROPE_HALF = 0
EBD_ROPE_PAIRS = 1
EBD_ROPE_INVERSE = 1

_P = ctypes.c_void_p
_BF = torch.bfloat16
_I32 = torch.int32


class ebd_rotary(ctypes.Structure):
    _fields_ = [
        ("freq", ctypes.c_void_p),
        ("rot_dim", ctypes.c_int32),
        ("layout", ctypes.c_int32),
        ("amplitude", ctypes.c_float),
        ("flags", ctypes.c_uint32),
    ]


class ebd_rows(ctypes.Structure):
    _fields_ = [("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class ebd_rope_params(ctypes.Structure):
    _fields_ = [
        ("num_tokens", ctypes.c_int32),
        ("num_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("x", ebd_rows),
        ("y", ebd_rows),
        ("pos", ctypes.c_void_p),
        ("rot", ebd_rotary),
    ]


class ebd_pages(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("max_pages", ctypes.c_int32),
        ("page_table", ctypes.c_void_p),
        ("page_stride", ctypes.c_int64),
        ("head_stride", ctypes.c_int64),
        ("row_stride", ctypes.c_int64),
    ]


class ebd_append_paged_params(ctypes.Structure):
    _fields_ = [
        ("pages", ebd_pages),
        ("num_tokens", ctypes.c_int64),
        ("new_off", ctypes.c_void_p),
        ("len", ctypes.c_void_p),
        ("pos", ctypes.c_void_p),
        ("rot", ebd_rotary),
        ("q_heads", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("k_rows", ebd_rows),
        ("v_rows", ebd_rows),
        ("q_rows", ebd_rows),
        ("q_out_rows", ebd_rows),
    ]


class ebd_attend_paged_params(ctypes.Structure):
    _fields_ = [
        ("pages", ebd_pages),
        ("group", ctypes.c_int32),
        ("max_new", ctypes.c_int32),
        ("num_tokens", ctypes.c_int64),
        ("max_rows", ctypes.c_int64),
        ("new_off", ctypes.c_void_p),
        ("len", ctypes.c_void_p),
        ("qpos", ctypes.c_void_p),
        ("window", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("q_rows", ebd_rows),
        ("y_rows", ebd_rows),
    ]


class ebd_gather_paged_params(ctypes.Structure):
    _fields_ = [
        ("pages", ebd_pages),
        ("max_rows", ctypes.c_int64),
        ("seq_off", ctypes.c_void_p),
        ("num_rows", ctypes.c_int64),
    ]


class ebd_attend_tree_params(ctypes.Structure):
    _fields_ = [
        ("attend", ebd_attend_paged_params),
        ("mask", ctypes.c_void_p),
        ("mask_words", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


class ebd_keep_rows_params(ctypes.Structure):
    _fields_ = [
        ("pages", ebd_pages),
        ("new_off", ctypes.c_void_p),
        ("len", ctypes.c_void_p),
        ("path", ctypes.c_void_p),
        ("kept", ctypes.c_void_p),
        ("len_out", ctypes.c_void_p),
        ("max_kept", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


class ebd_norm(ctypes.Structure):
    _fields_ = [
        ("weight", ctypes.c_void_p),
        ("head_stride", ctypes.c_int64),
        ("eps", ctypes.c_float),
        ("reserved", ctypes.c_int32),
    ]


class ebd_norm_rope_params(ctypes.Structure):
    _fields_ = [
        ("num_tokens", ctypes.c_int32),
        ("num_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("x", ebd_rows),
        ("y", ebd_rows),
        ("pos", ctypes.c_void_p),
        ("norm", ebd_norm),
        ("rot", ebd_rotary),
    ]


class ebd_norm_rope_backward_params(ctypes.Structure):
    _fields_ = [
        ("num_tokens", ctypes.c_int32),
        ("num_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("x", ebd_rows),
        ("dy", ebd_rows),
        ("dx", ebd_rows),
        ("pos", ctypes.c_void_p),
        ("norm", ebd_norm),
        ("rot", ebd_rotary),
    ]


class ebd_append_norm_params(ctypes.Structure):
    _fields_ = [
        ("append", ebd_append_paged_params),
        ("k_norm", ebd_norm),
        ("q_norm", ebd_norm),
        ("slots", ctypes.c_void_p),
    ]


class ebd_plan_step_params(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("max_pages", ctypes.c_int32),
        ("num_tokens", ctypes.c_int64),
        ("count", ctypes.c_void_p),
        ("len", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p),
        ("free_pages", ctypes.c_void_p),
        ("free_state", ctypes.c_void_p),
        ("new_off", ctypes.c_void_p),
        ("slots", ctypes.c_void_p),
        ("pos", ctypes.c_void_p),
        ("parent", ctypes.c_void_p),
        ("mask", ctypes.c_void_p),
        ("mask_words", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


_lib.ebd_rope.argtypes = [_P] * 4
_lib.ebd_rope.restype = ctypes.c_int
_lib.ebd_append_paged.argtypes = [_P] * 9
_lib.ebd_append_paged.restype = ctypes.c_int
_lib.ebd_attend_paged.argtypes = [_P] * 8 + [ctypes.c_size_t, _P]
_lib.ebd_attend_paged.restype = ctypes.c_int
_lib.ebd_gather_paged.argtypes = [_P] * 7
_lib.ebd_gather_paged.restype = ctypes.c_int
_lib.ebd_attend_tree.argtypes = [_P] * 8 + [ctypes.c_size_t, _P]
_lib.ebd_attend_tree.restype = ctypes.c_int
_lib.ebd_keep_rows.argtypes = [_P] * 5
_lib.ebd_keep_rows.restype = ctypes.c_int
_lib.ebd_norm_rope.argtypes = [_P] * 4
_lib.ebd_norm_rope.restype = ctypes.c_int
_lib.ebd_norm_rope_backward.argtypes = [_P] * 6 + [ctypes.c_size_t, _P]
_lib.ebd_norm_rope_backward.restype = ctypes.c_int
_lib.ebd_append_norm.argtypes = [_P] * 9
_lib.ebd_append_norm.restype = ctypes.c_int
_lib.ebd_plan_step.argtypes = [_P] * 3 + [ctypes.c_size_t, _P]
_lib.ebd_plan_step.restype = ctypes.c_int


# ---- tensors -> parameters ---------------------------------------------------------------------

def _table(t, dtype, shape, name):
    """Device pointer of a contiguous tensor of this type and shape."""
    p = _ptr(t, dtype, name)
    if t is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have the shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return p


def _here(*tensors):
    """The GPU that holds all of these tensors."""
    dev = None
    for t in tensors:
        if t is None:
            continue
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError("tensors of one call must be on one device: got %s and %s" % (dev, t.device))
    return dev


def _layout(t, name, heads=None, tokens=None):
    """(shape, strides) of rows [tokens, heads, 128] bf16, checked."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype != _BF:
        raise TypeError("%s must be %s, got %s" % (name, _BF, t.dtype))
    if t.dim() != 3 or t.shape[2] != HEAD_DIM or (t.numel() and t.stride(2) != 1):
        raise ValueError("%s must be [tokens, heads, %d] with contiguous rows" % (name, HEAD_DIM))
    if heads is not None and t.shape[1] != heads:
        raise ValueError("%s must have %d heads, got %d" % (name, heads, t.shape[1]))
    if tokens is not None and t.shape[0] != tokens:
        raise ValueError("%s must have %d tokens, got %d" % (name, tokens, t.shape[0]))
    return tuple(t.shape), t.stride()


def _rows_of(t):
    # a stride over one element is never used, and may be anything
    return ebd_rows(t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0)


def _distinct(t, name):
    """Refuse outputs whose rows may share memory: each stride has to pass over all that the smaller ones span."""
    span = HEAD_DIM
    for stride, n in sorted((s, n) for n, s in zip(t.shape[:-1], t.stride()[:-1]) if n > 1):
        if t.numel() and stride < span:
            raise ValueError("the rows of %s must not share memory" % name)
        span += stride * (n - 1)


def _plan(p, device, keep, **tensors):
    """Note what the calls on `p` must pass, and keep what its addresses point to."""
    if device.type != "cuda":
        raise ValueError("the tensors must be on the GPU")
    p.device, p.index, p.keep = device, device.index, keep
    p.expect = {n: None if t is None else (t.shape, t.stride()) for n, t in tensors.items()}
    p.at = ctypes.addressof(p)
    return p


# A call's checks cost as much host time as a small kernel runs, so that they read no more of a tensor than
# its type, device, shape and strides.

def _arg(p, name, t):
    """Address of a call's bf16 tensor, of the shape and strides the parameters were made for."""
    want = p.expect[name]
    if t is None and want is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if want is None:
        raise ValueError("%s: the parameters were made without it" % name)
    if t.dtype is not _BF:
        raise TypeError("%s must be %s, got %s" % (name, _BF, t.dtype))
    if t.get_device() != p.index:
        raise ValueError("%s must be on %s, got %s" % (name, p.device, t.device))
    if t.shape != want[0] or t.stride() != want[1]:
        raise ValueError("%s must have the shape and strides that the parameters were made for" % name)
    return t.data_ptr()


def _out(p, name, t, dtype, shape):
    """Address of an optional contiguous output of a call."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.get_device() != p.index:
        raise ValueError("%s must be on %s, got %s" % (name, p.device, t.device))
    if (shape is not None and t.shape != shape) or not t.is_contiguous():
        raise ValueError("%s must be contiguous%s" % (name, "" if shape is None else " and %s" % (tuple(shape),)))
    return t.data_ptr()


def _on_stream(p, stream):
    if p.index != torch._C._cuda_getDevice():
        raise ValueError("the tensors are on %s, which is not the current device" % p.device)
    return torch._C._cuda_getCurrentRawStream(p.index) if stream is None else stream.cuda_stream


def rotary(freq: Optional[torch.Tensor], layout: int = EBD_ROPE_HALF, amplitude: float = 1.0,
           inverse: bool = False) -> ebd_rotary:
    """Rotary positions by the frequencies `freq` [rot_dim / 2] (float64 radians per position)."""
    r = ebd_rotary()
    r.layout, r.amplitude = int(layout), float(amplitude)
    r.flags = EBD_ROPE_INVERSE if inverse else 0
    if freq is not None:
        r.freq = _ptr(freq, torch.float64, "freq")
        if freq.dim() != 1 or not 1 <= freq.numel() <= HEAD_DIM // 2:
            raise ValueError("freq must be [rot_dim / 2], 1 to %d of them" % (HEAD_DIM // 2))
        r.rot_dim = 2 * freq.numel()
    r.keep = freq
    return r


def rope_params(x, y, pos, rot: ebd_rotary) -> ebd_rope_params:
    """Rows x [tokens, heads, 128] -> y (may be x), pos [tokens] int32."""
    (tokens, heads, _), _ = _layout(x, "x")
    _layout(y, "y", heads, tokens)
    _distinct(y, "y")
    if rot.keep is None:
        raise ValueError("rope needs frequencies")
    p = ebd_rope_params()
    p.num_tokens, p.num_heads, p.head_dim = tokens, heads, HEAD_DIM
    p.x, p.y = _rows_of(x), _rows_of(y)
    p.pos = _table(pos, torch.int32, (tokens,), "pos")
    p.rot = rot
    return _plan(p, _here(x, y, pos, rot.keep), (pos, rot.keep), x=x, y=y)


def head_norm(weight, eps: float = 1e-6) -> ebd_norm:
    """Norms of heads: weights [128] of all heads, or [heads, 128] of each one's own (fp32; one row expanded over the heads
    serves forward calls only)."""
    if not isinstance(weight, torch.Tensor):
        raise TypeError("weight must be a torch.Tensor")
    if weight.dtype != torch.float32:
        raise TypeError("weight must be %s, got %s" % (torch.float32, weight.dtype))
    if weight.device.type != "cuda":
        raise ValueError("weight must be on the GPU")
    if weight.dim() not in (1, 2) or weight.shape[-1] != HEAD_DIM or weight.stride(-1) != 1:
        raise ValueError("weight must be [%d] or [heads, %d] with contiguous rows" % (HEAD_DIM, HEAD_DIM))
    n = ebd_norm()
    n.weight, n.eps = weight.data_ptr(), float(eps)
    if weight.dim() == 2:  # (a stride over one head is never used, and may be anything)
        n.head_stride = weight.stride(0) if weight.shape[0] > 1 else HEAD_DIM
    n.keep = weight
    return n


def _norm_of(norm, heads, name):
    if not isinstance(norm, ebd_norm):
        raise TypeError("%s must be made by head_norm" % name)
    if norm.keep.dim() == 2 and norm.keep.shape[0] != heads:
        raise ValueError("%s has weights of %d heads, not %d" % (name, norm.keep.shape[0], heads))
    return norm


def _turned(p, rot, pos, tokens):
    """Note a rotation (or none) and its positions; returns the frequencies."""
    if rot is None:
        return None
    if rot.keep is None:
        raise ValueError("rot needs frequencies")
    if pos is None:
        raise ValueError("a rotation needs positions")
    p.rot = rot
    p.pos = _table(pos, torch.int32, (tokens,), "pos")
    return rot.keep


def norm_rope_params(x, y, norm: ebd_norm, rot: Optional[ebd_rotary] = None, pos=None) -> ebd_norm_rope_params:
    """Rows x [tokens, heads, 128] -> y (may be x), normalised, and with `rot` rotated by pos [tokens] int32."""
    (tokens, heads, _), _ = _layout(x, "x")
    _layout(y, "y", heads, tokens)
    _distinct(y, "y")
    p = ebd_norm_rope_params()
    p.num_tokens, p.num_heads, p.head_dim = tokens, heads, HEAD_DIM
    p.x, p.y = _rows_of(x), _rows_of(y)
    p.norm = _norm_of(norm, heads, "norm")
    freq = _turned(p, rot, pos, tokens)
    return _plan(p, _here(x, y, pos if rot else None, norm.keep, freq), (pos, norm.keep, freq), x=x, y=y)


def norm_rope_backward_params(x, dy, dx, norm: ebd_norm, rot: Optional[ebd_rotary] = None,
                              pos=None) -> ebd_norm_rope_backward_params:
    """Gradients of norm_rope_params' call with the same norm, rot and pos: dy -> dx (may be dy or x)."""
    if isinstance(norm, ebd_norm) and norm.keep.dim() == 2 and norm.head_stride == 0:
        # (the heads' gradients would be added up in the first row, and the others left as they were)
        raise ValueError("norm has one row of weights, expanded over the heads: give head_norm that row")
    (tokens, heads, _), _ = _layout(x, "x")
    _layout(dy, "dy", heads, tokens)
    _layout(dx, "dx", heads, tokens)
    _distinct(dx, "dx")
    p = ebd_norm_rope_backward_params()
    p.num_tokens, p.num_heads, p.head_dim = tokens, heads, HEAD_DIM
    p.x, p.dy, p.dx = _rows_of(x), _rows_of(dy), _rows_of(dx)
    p.norm = _norm_of(norm, heads, "norm")
    freq = _turned(p, rot, pos, tokens)
    p.weights = norm.keep.shape
    return _plan(p, _here(x, dy, dx, pos if rot else None, norm.keep, freq), (pos, norm.keep, freq), x=x, dy=dy, dx=dx)


def append_norm_params(pgs: ebd_pages, k_new, v_new, new_off=None, len=None, k_norm: Optional[ebd_norm] = None,
                       q_norm: Optional[ebd_norm] = None, rot: Optional[ebd_rotary] = None, pos=None, q=None, q_out=None,
                       slots=None) -> ebd_append_norm_params:
    """As append_paged_params, the keys normalised by k_norm and the queries by q_norm (None: not).  With slots [tokens]
    int64 (of ebd_plan_step) the tokens go there: new_off and len are not needed, and a rotation needs pos."""
    (tokens, _, _), _ = _layout(k_new, "k_new", pgs.kv_heads)
    if slots is not None and rot is not None and pos is None:
        raise ValueError("with slots, a rotation needs positions")
    if slots is None and (new_off is None or len is None):
        raise ValueError("without slots, new_off and len are needed")
    a = append_paged_params(pgs, k_new, v_new, new_off, len, rot, pos=pos, q=q, q_out=q_out)
    p = ebd_append_norm_params()
    p.append = a
    if k_norm is not None:
        p.k_norm = _norm_of(k_norm, pgs.kv_heads, "k_norm")
    if q_norm is not None:
        if q is None:
            raise ValueError("q_norm goes with q")
        p.q_norm = _norm_of(q_norm, q.shape[1], "q_norm")
    p.slots = _table(slots, torch.int64, (tokens,), "slots")
    w = [n.keep for n in (k_norm, q_norm) if n is not None]
    dev = _here(pgs.pools[0], slots, *w)
    _plan(p, dev, (a.keep, slots, *w))
    p.expect, p.seqs = a.expect, a.seqs
    return p


def pages(K, V, page_table) -> ebd_pages:
    """The pools K and V [pages, KV heads, rows per page, 128] (any strides over the first three, the same
    for both) and page_table [sequences, pages per sequence] int32."""
    for t, name in ((K, "K"), (V, "V")):
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a torch.Tensor" % name)
        if t.dtype != _BF:
            raise TypeError("%s must be %s, got %s" % (name, _BF, t.dtype))
        if t.dim() != 4 or t.shape[3] != HEAD_DIM or t.stride(3) != 1:
            raise ValueError("%s must be [pages, KV heads, rows, %d] with contiguous rows" % (name, HEAD_DIM))
    if K.shape != V.shape or K.stride() != V.stride():
        raise ValueError("K and V must have the same shape and strides")
    _distinct(K, "K")
    table = _ptr(page_table, torch.int32, "page_table")
    if page_table is None or page_table.dim() != 2:
        raise ValueError("page_table must be [sequences, pages per sequence]")
    P = ebd_pages()
    P.num_pages, P.kv_heads, P.page_size, P.head_dim = *K.shape[:3], HEAD_DIM
    P.num_seqs, P.max_pages = page_table.shape
    P.page_table = table
    # strides over one page, head or row are never used, and may be anything
    P.page_stride, P.head_stride, P.row_stride = (s if n > 1 else HEAD_DIM
                                                  for n, s in zip(K.shape[:3], K.stride()[:3]))
    P.pools, P.keep = (K, V), page_table
    return P


def append_paged_params(pgs: ebd_pages, k_new, v_new, new_off, len, rot: Optional[ebd_rotary] = None,
                        pos=None, q=None, q_out=None) -> ebd_append_paged_params:
    """New tokens k_new, v_new [tokens, KV heads, 128] (and q -> q_out [tokens, query heads, 128]) of the
    sequences new_off [sequences + 1] int64, which hold len [sequences] int32 rows with them.  rot None:
    nothing is rotated; pos [tokens] int32 None: a token's position is its row."""
    (tokens, _, _), _ = _layout(k_new, "k_new", pgs.kv_heads)
    _layout(v_new, "v_new", pgs.kv_heads, tokens)
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    p = ebd_append_paged_params()
    p.pages, p.num_tokens = pgs, tokens
    p.new_off = _table(new_off, torch.int64, (pgs.num_seqs + 1,), "new_off")
    p.len = _table(len, torch.int32, (pgs.num_seqs,), "len")
    p.pos = _table(pos, torch.int32, (tokens,), "pos")
    freq = None
    if rot is not None:
        p.rot, freq = rot, rot.keep
    p.k_rows, p.v_rows = _rows_of(k_new), _rows_of(v_new)
    if q is not None:
        (_, heads, _), _ = _layout(q, "q", None, tokens)
        _layout(q_out, "q_out", heads, tokens)
        _distinct(q_out, "q_out")
        p.q_heads, p.q_rows, p.q_out_rows = heads, _rows_of(q), _rows_of(q_out)
    K, V = pgs.pools
    p.seqs = (pgs.num_seqs,)
    dev = _here(K, V, pgs.keep, k_new, v_new, new_off, len, pos, freq, q, q_out)
    return _plan(p, dev, (pgs.keep, new_off, len, pos, freq), K=K, V=V, k_new=k_new, v_new=v_new, q=q, q_out=q_out)


def attend_paged_params(pgs: ebd_pages, q, y, new_off, len, max_new: int, max_rows: int, qpos=None,
                        window: int = 0, scale: float = 0.0) -> ebd_attend_paged_params:
    """Queries q -> y [tokens, query heads, 128] of the sequences new_off [sequences + 1] int64 (at most
    max_new tokens each), which hold len [sequences] int32 rows (at most max_rows)."""
    (tokens, heads, _), _ = _layout(q, "q")
    _layout(y, "y", heads, tokens)
    _distinct(y, "y")
    if heads < 1 or heads % pgs.kv_heads:
        raise ValueError("query heads (%d) must be a multiple of the KV heads (%d)" % (heads, pgs.kv_heads))
    p = ebd_attend_paged_params()
    p.pages, p.num_tokens, p.group = pgs, tokens, heads // pgs.kv_heads
    p.max_new, p.max_rows = int(max_new), int(max_rows)
    p.new_off = _table(new_off, torch.int64, (pgs.num_seqs + 1,), "new_off")
    p.len = _table(len, torch.int32, (pgs.num_seqs,), "len")
    p.qpos = _table(qpos, torch.int32, (tokens,), "qpos")
    p.window, p.scale = int(window), float(scale)
    p.q_rows, p.y_rows = _rows_of(q), _rows_of(y)
    p.seqs, p.heads = (pgs.num_seqs,), (tokens, heads)
    K, V = pgs.pools
    return _plan(p, _here(K, V, pgs.keep, q, y, new_off, len, qpos), (pgs.keep, new_off, len, qpos),
                 K=K, V=V, q=q, y=y)


def attend_tree_params(pgs: ebd_pages, q, y, new_off, len, max_new: int, max_rows: int, mask, qpos=None,
                       window: int = 0, scale: float = 0.0) -> ebd_attend_tree_params:
    """As attend_paged_params, but new tokens see each other by mask [tokens, words] int64: bit i of word w is the
    sequence's new token 64 w + i.  qpos (positions) then serve the window alone, over the rows held before."""
    a = attend_paged_params(pgs, q, y, new_off, len, max_new, max_rows, qpos=qpos, window=window, scale=scale)
    if not isinstance(mask, torch.Tensor) or mask.dim() != 2:
        raise ValueError("mask must be [tokens, words]")
    p = ebd_attend_tree_params()
    p.attend = a
    p.mask, p.mask_words = _table(mask, torch.int64, (q.shape[0], mask.shape[1]), "mask"), mask.shape[1]
    _plan(p, _here(q, mask), (a.keep, mask))
    p.expect, p.seqs, p.heads = a.expect, a.seqs, a.heads
    return p


def keep_rows_params(pgs: ebd_pages, new_off, len, path, kept, len_out=None) -> ebd_keep_rows_params:
    """Of sequences new_off [sequences + 1] int64 that hold len [sequences] int32 rows, the new tokens path [sequences,
    most kept] int32 (the first kept [sequences] int32 of each) are kept; len_out [sequences] int32 (may be len) receives
    the rows then held."""
    S = pgs.num_seqs
    if not isinstance(path, torch.Tensor) or path.dim() != 2:
        raise ValueError("path must be [sequences, most kept]")
    p = ebd_keep_rows_params()
    p.pages, p.max_kept = pgs, path.shape[1]
    p.new_off, p.len = _table(new_off, torch.int64, (S + 1,), "new_off"), _table(len, _I32, (S,), "len")
    p.path, p.kept = _table(path, _I32, (S, path.shape[1]), "path"), _table(kept, _I32, (S,), "kept")
    p.len_out = _table(len_out, _I32, (S,), "len_out")
    p.seqs = (S,)
    K, V = pgs.pools
    return _plan(p, _here(K, V, pgs.keep, new_off, len, path, kept, len_out), (pgs.keep, new_off, len, path, kept, len_out),
                 K=K, V=V)


def gather_paged_params(pgs: ebd_pages, seq_off, max_rows: int) -> ebd_gather_paged_params:
    """Units seq_off [sequences * KV heads + 1] int64, the longest at most max_rows.  The rows that there is room for
    are those of each call's outputs."""
    p = ebd_gather_paged_params()
    p.pages, p.max_rows = pgs, int(max_rows)
    p.seq_off = _table(seq_off, torch.int64, (pgs.num_seqs * pgs.kv_heads + 1,), "seq_off")
    p.units = (pgs.num_seqs * pgs.kv_heads,)
    K, V = pgs.pools
    return _plan(p, _here(K, V, pgs.keep, seq_off), (pgs.keep, seq_off), K=K, V=V)


def plan_step_params(count, len, page_table, page_size: int, free_pages, free_state, new_off, slots=None, pos=None,
                     parent=None, mask=None) -> ebd_plan_step_params:
    """New tokens count [sequences] int32 (negative: ended) of sequences that hold len [sequences] int32 rows in the pages
    page_table [sequences, pages per sequence] int32; free_pages [pages of the pool] int32, a ring, and free_state [2] int32.
    Written: new_off [sequences + 1] int64, slots [tokens] int64, pos [tokens] int32; with the trees parent [tokens] int32
    also mask [tokens, words] int64.  len, page_table, free_pages and free_state are updated."""
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be [sequences, pages per sequence]")
    if not isinstance(free_pages, torch.Tensor) or free_pages.dim() != 1 or free_pages.numel() < 1:
        raise ValueError("free_pages must be [pages of the pool]")
    if (parent is None) != (mask is None):
        raise ValueError("parent and mask go together")
    S = page_table.shape[0]
    room = {t.shape[0] for t in (slots, pos, parent, mask) if isinstance(t, torch.Tensor) and t.dim()}
    if builtins.len(room) > 1:
        raise ValueError("slots, pos, parent and mask must have the same number of tokens")
    p = ebd_plan_step_params()
    p.num_seqs, p.max_pages = page_table.shape
    p.page_size, p.num_pages, p.num_tokens = int(page_size), free_pages.numel(), room.pop() if room else 0
    T = (p.num_tokens,)
    p.count, p.len = _table(count, _I32, (S,), "count"), _table(len, _I32, (S,), "len")
    p.page_table = _table(page_table, _I32, page_table.shape, "page_table")
    p.free_pages = _table(free_pages, _I32, free_pages.shape, "free_pages")
    p.free_state, p.new_off = _table(free_state, _I32, (2,), "free_state"), _table(new_off, torch.int64, (S + 1,), "new_off")
    p.slots, p.pos = _table(slots, torch.int64, T, "slots"), _table(pos, _I32, T, "pos")
    if mask is not None:
        if not isinstance(mask, torch.Tensor) or mask.dim() != 2:
            raise ValueError("mask must be [tokens, words]")
        p.parent, p.mask = _table(parent, _I32, T, "parent"), _table(mask, torch.int64, mask.shape, "mask")
        p.mask_words = mask.shape[1]
    p.seqs = (S,)
    held = (count, len, page_table, free_pages, free_state, new_off, slots, pos, parent, mask)
    return _plan(p, _here(*held), held)


# ---- the calls ---------------------------------------------------------------------------------

def ebd_rope(params: ebd_rope_params, x, y, stream=None) -> None:
    """Rotate rows x into y (asynchronous on the current stream)."""
    code = _lib.ebd_rope(params.at, _arg(params, "x", x), _arg(params, "y", y), _on_stream(params, stream))
    _check("ebd_rope", code)


def ebd_append_paged(params: ebd_append_paged_params, k_new, v_new, K, V, q=None, q_out=None, status=None,
                     stream=None) -> None:
    """Write new tokens into their pages, and rotate their queries (asynchronous)."""
    code = _lib.ebd_append_paged(params.at, _arg(params, "k_new", k_new), _arg(params, "v_new", v_new),
                                 _arg(params, "K", K), _arg(params, "V", V), _arg(params, "q", q),
                                 _arg(params, "q_out", q_out), _out(params, "status", status, _I32, params.seqs),
                                 _on_stream(params, stream))
    _check("ebd_append_paged", code)


def ebd_attend_paged(params: ebd_attend_paged_params, q, K, V, y, workspace, lse=None, status=None,
                     stream=None) -> None:
    """Attention of the new tokens over the paged cache (asynchronous)."""
    if not isinstance(workspace, torch.Tensor):
        raise TypeError("workspace must be a torch.Tensor")
    code = _lib.ebd_attend_paged(params.at, _arg(params, "q", q), _arg(params, "K", K), _arg(params, "V", V),
                                 _arg(params, "y", y), _out(params, "lse", lse, torch.float32, params.heads),
                                 _out(params, "status", status, _I32, params.seqs),
                                 _out(params, "workspace", workspace, workspace.dtype, None), workspace.nbytes,
                                 _on_stream(params, stream))
    _check("ebd_attend_paged", code)


def ebd_attend_tree(params: ebd_attend_tree_params, q, K, V, y, workspace, lse=None, status=None, stream=None) -> None:
    """Attention of trees of drafted tokens over the paged cache (asynchronous)."""
    if not isinstance(workspace, torch.Tensor):
        raise TypeError("workspace must be a torch.Tensor")
    code = _lib.ebd_attend_tree(params.at, _arg(params, "q", q), _arg(params, "K", K), _arg(params, "V", V),
                                _arg(params, "y", y), _out(params, "lse", lse, torch.float32, params.heads),
                                _out(params, "status", status, _I32, params.seqs),
                                _out(params, "workspace", workspace, workspace.dtype, None), workspace.nbytes,
                                _on_stream(params, stream))
    _check("ebd_attend_tree", code)


def ebd_keep_rows(params: ebd_keep_rows_params, K, V, status=None, stream=None) -> None:
    """Move the rows of the accepted paths together (asynchronous)."""
    code = _lib.ebd_keep_rows(params.at, _arg(params, "K", K), _arg(params, "V", V),
                              _out(params, "status", status, _I32, params.seqs), _on_stream(params, stream))
    _check("ebd_keep_rows", code)


def ebd_gather_paged(params: ebd_gather_paged_params, K, V, Ku, Vu, status=None, stream=None) -> None:
    """Read the pages out as units Ku, Vu [rows, 128], of the same size (asynchronous)."""
    ku, vu = _out(params, "Ku", Ku, _BF, None), _out(params, "Vu", Vu, _BF, None)
    shape = None if Ku is None else Ku.shape
    if shape is None or Vu is None or len(shape) != 2 or shape[1] != HEAD_DIM or Vu.shape != shape:
        raise ValueError("Ku and Vu must both be [rows, %d]" % HEAD_DIM)
    p = ebd_gather_paged_params.from_buffer_copy(params)  # (of this call: calls on the same parameters may overlap)
    p.num_rows = shape[0]
    code = _lib.ebd_gather_paged(ctypes.addressof(p), _arg(params, "K", K), _arg(params, "V", V), ku, vu,
                                 _out(params, "status", status, _I32, params.units), _on_stream(params, stream))
    _check("ebd_gather_paged", code)


def ebd_norm_rope(params: ebd_norm_rope_params, x, y, stream=None) -> None:
    """Normalise and rotate rows x into y (asynchronous)."""
    code = _lib.ebd_norm_rope(params.at, _arg(params, "x", x), _arg(params, "y", y), _on_stream(params, stream))
    _check("ebd_norm_rope", code)


def ebd_norm_rope_backward(params: ebd_norm_rope_backward_params, x, dy, dx, dweight, workspace, stream=None) -> None:
    """Gradients dx and dweight (fp32, the weights' shape, contiguous) of ebd_norm_rope (asynchronous)."""
    if not isinstance(dweight, torch.Tensor):
        raise TypeError("dweight must be a torch.Tensor")
    if not isinstance(workspace, torch.Tensor):
        raise TypeError("workspace must be a torch.Tensor")
    code = _lib.ebd_norm_rope_backward(params.at, _arg(params, "x", x), _arg(params, "dy", dy), _arg(params, "dx", dx),
                                       _out(params, "dweight", dweight, torch.float32, params.weights),
                                       _out(params, "workspace", workspace, workspace.dtype, None), workspace.nbytes,
                                       _on_stream(params, stream))
    _check("ebd_norm_rope_backward", code)


def ebd_append_norm(params: ebd_append_norm_params, k_new, v_new, K, V, q=None, q_out=None, status=None,
                    stream=None) -> None:
    """Write new tokens into their pages, keys and queries normalised and rotated (asynchronous)."""
    code = _lib.ebd_append_norm(params.at, _arg(params, "k_new", k_new), _arg(params, "v_new", v_new),
                                _arg(params, "K", K), _arg(params, "V", V), _arg(params, "q", q),
                                _arg(params, "q_out", q_out), _out(params, "status", status, _I32, params.seqs),
                                _on_stream(params, stream))
    _check("ebd_append_norm", code)


def ebd_plan_step(params: ebd_plan_step_params, workspace, status=None, stream=None) -> None:
    """Pages, offsets, slots, positions and masks of a step (asynchronous)."""
    if not isinstance(workspace, torch.Tensor):
        raise TypeError("workspace must be a torch.Tensor")
    code = _lib.ebd_plan_step(params.at, _out(params, "status", status, _I32, params.seqs),
                              _out(params, "workspace", workspace, workspace.dtype, None), workspace.nbytes,
                              _on_stream(params, stream))
    _check("ebd_plan_step", code)


# ---- helpers that allocate ---------------------------------------------------------------------

def rope_frequencies(rot_dim: int = HEAD_DIM, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     original: int = 0, low: Optional[float] = None, high: Optional[float] = None, device="cuda"):
    """(frequencies [rot_dim / 2] float64, amplitude) of f_i = base^(-2i / rot_dim), scaled for contexts `factor` times
    as long as the `original` ones:

      none    as they are
      linear  f / factor (positions interpolated)
      ntk     base -> base factor^(rot_dim / (rot_dim - 2)): the highest frequency stays, the lowest becomes f / factor
      bands   by the turns t = original f / 2 pi that a pair makes over the original context: f from `high` turns
              (default 4) on, f / factor up to `low` (default 1), and between them g f + (1 - g) f / factor with
              g = (t - low) / (high - low)
      yarn    as bands, with `high` 32, and the amplitude 0.1 ln(factor) + 1: linear in the turns, as the method is
              written.  Checkpoints whose frequencies were blended linearly in the pair's index i, between the (perhaps
              rounded) indices at which the turns are `high` and `low`, were trained with others in that band: give
              `rotary` those.
    """
    if rot_dim < 2 or rot_dim > HEAD_DIM or rot_dim % 2:
        raise ValueError("rot_dim must be even, 2 to %d" % HEAD_DIM)
    if not (base > 0 and factor > 0 and math.isfinite(base) and math.isfinite(factor)):
        raise ValueError("base and factor must be positive")
    amplitude = 1.0
    if scaling == "ntk":
        if rot_dim == 2:
            raise ValueError("ntk scaling needs more than one pair")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-2.0 * torch.arange(rot_dim // 2, dtype=torch.float64) / rot_dim)
    if scaling == "linear":
        f = f / factor
    elif scaling in ("bands", "yarn"):
        low = 1.0 if low is None else low
        high = (32.0 if scaling == "yarn" else 4.0) if high is None else high
        if original < 1 or not low < high:
            raise ValueError("%s scaling needs the original context length, and low < high" % scaling)
        g = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        f = g * f + (1 - g) * f / factor
        if scaling == "yarn" and factor > 1:
            amplitude = 0.1 * math.log(factor) + 1.0
    elif scaling not in ("none", "ntk"):
        raise ValueError("unknown scaling %r" % (scaling,))
    return f.to(device), amplitude


@dataclass
class PagedCache:
    """The pools of one layer and what its sequences hold: K, V [pages, KV heads, rows per page, 128] bf16, page_table
    [sequences, pages per sequence] int32, len [sequences] int32 (all on the device, the caller's to update).  A pool whose
    pages `plan` deals out has its free ones in the ring free_pages [pages] int32, free_state [2] int32.  The layers of a model
    are caches with pools of their own that share page_table and len: one of them plans a step, and the last one's `keep`
    updates len."""

    K: torch.Tensor
    V: torch.Tensor
    page_table: torch.Tensor
    len: torch.Tensor
    free_pages: Optional[torch.Tensor] = None
    free_state: Optional[torch.Tensor] = None

    @classmethod
    def allocate(cls, lengths: Sequence[int], kv_heads: int, page_size: int = 64, spare: int = 0, device="cuda"):
        """A pool with room for `lengths` rows of each sequence (and `spare` pages), tables filled, len zero."""
        used = [-(-max(int(n), 0) // page_size) for n in lengths]
        total = max(sum(used) + spare, 1)
        table = torch.full((len(used), max(used, default=0) or 1), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(used):
            table[s, :n] = torch.arange(at, at + n, dtype=torch.int32)
            at += n
        shape = (total, kv_heads, page_size, HEAD_DIM)
        return cls(torch.empty(shape, dtype=_BF, device=device), torch.empty(shape, dtype=_BF, device=device),
                   table.to(device), torch.zeros(len(used), dtype=torch.int32, device=device))

    @classmethod
    def pool(cls, num_seqs: int, num_pages: int, kv_heads: int, page_size: int = 64, max_pages: Optional[int] = None,
             device="cuda"):
        """A pool of free pages and `num_seqs` sequences without rows, of up to max_pages pages each (default: all)."""
        shape = (num_pages, kv_heads, page_size, HEAD_DIM)
        table = torch.full((num_seqs, num_pages if max_pages is None else max_pages), -1, dtype=torch.int32, device=device)
        return cls(torch.empty(shape, dtype=_BF, device=device), torch.empty(shape, dtype=_BF, device=device), table,
                   torch.zeros(num_seqs, dtype=torch.int32, device=device),
                   torch.arange(num_pages, dtype=torch.int32, device=device),
                   torch.tensor([0, num_pages], dtype=torch.int32, device=device))

    @property
    def pages(self) -> ebd_pages:
        return pages(self.K, self.V, self.page_table)

    def plan(self, count, num_tokens: int, parent=None, mask_words: Optional[int] = None, ws: Optional[torch.Tensor] = None,
             status=None):
        """Pages for the new tokens count [sequences] int32 (negative: the sequence has ended) of a step of at most
        num_tokens tokens, and len with them: {"new_off", "slots" [num_tokens] int64, "pos" [num_tokens] int32, "ws"}, and
        with the trees parent [num_tokens] int32 "mask" [num_tokens, mask_words] int64 (by default of as many words as
        num_tokens tokens need, up to 64)."""
        if self.free_pages is None or self.free_state is None:
            raise ValueError("the cache has no ring of free pages")
        dev, T = self.K.device, int(num_tokens)
        new = {"new_off": torch.empty(self.len.numel() + 1, dtype=torch.int64, device=dev),
               "slots": torch.empty(T, dtype=torch.int64, device=dev), "pos": torch.empty(T, dtype=_I32, device=dev)}
        if parent is not None:
            words = max(1, min(64, -(-T // 64))) if mask_words is None else int(mask_words)
            new["mask"] = torch.empty((T, words), dtype=torch.int64, device=dev)
        p = plan_step_params(count, self.len, self.page_table, self.K.shape[2], self.free_pages, self.free_state,
                             new["new_off"], slots=new["slots"], pos=new["pos"], parent=parent, mask=new.get("mask"))
        need = ebd_workspace_size(EBD_WS_PLAN_STEP, p)
        new["ws"] = workspace(need, dev) if ws is None or ws.numel() < need else ws
        ebd_plan_step(p, new["ws"], status=status)
        return new

    def append(self, k_new, v_new, new_off, rot: Optional[ebd_rotary] = None, pos=None, q=None, status=None,
               k_norm: Optional[ebd_norm] = None, q_norm: Optional[ebd_norm] = None, slots=None):
        """Append tokens (self.len counts them already), normalised by k_norm and q_norm, at their slots if given (of
        `plan`; a rotation then needs pos); returns the queries as the attention takes them (zeros for padding tokens), or
        None without q."""
        q_out = None if q is None else torch.zeros(q.shape, dtype=_BF, device=q.device)
        if k_norm is None and q_norm is None and slots is None:
            p = append_paged_params(self.pages, k_new, v_new, new_off, self.len, rot, pos=pos, q=q, q_out=q_out)
            ebd_append_paged(p, k_new, v_new, self.K, self.V, q, q_out, status=status)
        else:
            p = append_norm_params(self.pages, k_new, v_new, new_off, self.len, k_norm, q_norm, rot, pos=pos, q=q,
                                   q_out=q_out, slots=slots)
            ebd_append_norm(p, k_new, v_new, self.K, self.V, q, q_out, status=status)
        return q_out

    def attend(self, q, new_off, max_new: int, max_rows: int, qpos=None, window: int = 0, scale: float = 0.0,
               ws: Optional[torch.Tensor] = None, status=None):
        """Attention of the new tokens: {"y" [tokens, heads, 128] bf16, "lse" [tokens, heads] fp32, "ws"}; zeros and -inf
        for padding tokens and those past max_new."""
        y = torch.zeros(q.shape, dtype=_BF, device=q.device)
        lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float32, device=q.device)
        p = attend_paged_params(self.pages, q, y, new_off, self.len, max_new, max_rows, qpos=qpos, window=window,
                                scale=scale)
        need = ebd_workspace_size(EBD_WS_ATTEND_PAGED, p)
        if ws is None or ws.numel() < need:
            ws = workspace(need, q.device)
        ebd_attend_paged(p, q, self.K, self.V, y, ws, lse=lse, status=status)
        return {"y": y, "lse": lse, "ws": ws}

    def attend_tree(self, q, new_off, max_new: int, max_rows: int, mask, qpos=None, window: int = 0, scale: float = 0.0,
                    ws: Optional[torch.Tensor] = None, status=None):
        """Attention of trees of new tokens, as `attend`; mask and qpos as `plan` makes them."""
        y = torch.zeros(q.shape, dtype=_BF, device=q.device)
        lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float32, device=q.device)
        p = attend_tree_params(self.pages, q, y, new_off, self.len, max_new, max_rows, mask, qpos=qpos, window=window,
                               scale=scale)
        need = ebd_workspace_size(EBD_WS_ATTEND_TREE, p)
        if ws is None or ws.numel() < need:
            ws = workspace(need, q.device)
        ebd_attend_tree(p, q, self.K, self.V, y, ws, lse=lse, status=status)
        return {"y": y, "lse": lse, "ws": ws}

    def keep(self, new_off, path, kept, status=None, update_len: bool = True):
        """Keep the accepted paths path [sequences, most kept] int32 of kept [sequences] int32 tokens; len then counts
        these alone.  Layers whose caches share len (and the table, of one plan) find their rows by it: all but the last one's
        call need update_len False, which leaves it as it is."""
        p = keep_rows_params(self.pages, new_off, self.len, path, kept, len_out=self.len if update_len else None)
        ebd_keep_rows(p, self.K, self.V, status=status)

    def gather(self, lengths: Sequence[int], status=None):
        """The first lengths[s] rows of every sequence as units: (K [rows, 128], V, seq_off), as cache.evict takes them
        with the unit lengths [n for n in lengths for each KV head]."""
        off = [0]
        for n in lengths:
            off += [off[-1] + int(n) * (i + 1) for i in range(self.K.shape[1])]
        seq_off = torch.tensor(off, dtype=torch.int64, device=self.K.device)
        K = torch.empty((max(off[-1], 1), HEAD_DIM), dtype=_BF, device=self.K.device)
        V = torch.empty_like(K)
        p = gather_paged_params(self.pages, seq_off, max(lengths, default=0))
        ebd_gather_paged(p, self.K, self.V, K, V, status=status)
        return K, V, seq_off
