"""The paged cache in front of the eviction: binding and helpers (no method arithmetic).

    ebd_rope            rotary positions of query or key rows
    ebd_append_paged    new tokens into their sequences' pages, keys rotated on the way, queries too
    ebd_attend_paged    attention of a chunk of new tokens, or of a decode step, over the pages
    ebd_gather_paged    the pages read out as units, which ebd_scores and ebd_evict take

Each call takes a parameter struct (`rope_params`, `append_paged_params`, ...) that a program makes once
per plan and keeps: it holds the tables' addresses and the rows' strides.  A struct keeps the tensors
whose addresses it holds alive, and the tensors of a call must have the shapes and strides it was made for.
`PagedCache` holds a pool and makes the structs and outputs of each call; `rope_frequencies` gives the
frequencies of the usual rotary positions.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import EBD_WS_ATTEND_PAGED, HEAD_DIM, _check, _lib, _ptr, ebd_workspace_size, workspace

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


_lib.ebd_rope.argtypes = [_P] * 4
_lib.ebd_rope.restype = ctypes.c_int
_lib.ebd_append_paged.argtypes = [_P] * 9
_lib.ebd_append_paged.restype = ctypes.c_int
_lib.ebd_attend_paged.argtypes = [_P] * 8 + [ctypes.c_size_t, _P]
_lib.ebd_attend_paged.restype = ctypes.c_int
_lib.ebd_gather_paged.argtypes = [_P] * 7
_lib.ebd_gather_paged.restype = ctypes.c_int


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


def gather_paged_params(pgs: ebd_pages, seq_off, max_rows: int) -> ebd_gather_paged_params:
    """Units seq_off [sequences * KV heads + 1] int64, the longest at most max_rows.  The rows that there is room for
    are those of each call's outputs."""
    p = ebd_gather_paged_params()
    p.pages, p.max_rows = pgs, int(max_rows)
    p.seq_off = _table(seq_off, torch.int64, (pgs.num_seqs * pgs.kv_heads + 1,), "seq_off")
    p.units = (pgs.num_seqs * pgs.kv_heads,)
    K, V = pgs.pools
    return _plan(p, _here(K, V, pgs.keep, seq_off), (pgs.keep, seq_off), K=K, V=V)


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
    [sequences, pages per sequence] int32, len [sequences] int32 (all on the device, the caller's to update)."""

    K: torch.Tensor
    V: torch.Tensor
    page_table: torch.Tensor
    len: torch.Tensor

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

    @property
    def pages(self) -> ebd_pages:
        return pages(self.K, self.V, self.page_table)

    def append(self, k_new, v_new, new_off, rot: Optional[ebd_rotary] = None, pos=None, q=None, status=None):
        """Append tokens (self.len counts them already); returns the rotated queries (zeros for padding tokens), or None
        without q."""
        q_out = None if q is None else torch.zeros(q.shape, dtype=_BF, device=q.device)
        p = append_paged_params(self.pages, k_new, v_new, new_off, self.len, rot, pos=pos, q=q, q_out=q_out)
        ebd_append_paged(p, k_new, v_new, self.K, self.V, q, q_out, status=status)
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
