"""ctypes binding of the paged-cache calls of liblsm_index.so (include/lsm_cache.h; same names as the C entry points).

Tensors are torch tensors on the GPU:
  q, k, v          [n_tokens, heads, head_dim], any strides with contiguous elements of a head; bfloat16, float16 (or float32,
                   not for attention)
  k_pages, v_pages [n_pages, page_tokens, kv_heads, head_dim], any strides likewise: a layer's slice of blocks that hold all
                   layers' keys and values is fine
  positions, page tables, lengths, offsets   int32, contiguous;  slots   int64, contiguous
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from .binding import LsmError, _load, _stream_ptr

_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


class _Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("heads", C.c_uint64)]


class _Pages(C.Structure):
    _fields_ = [("data", C.c_void_p), ("page_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class _Rotation(C.Structure):
    _fields_ = [("positions", C.c_void_p), ("table", C.c_void_p), ("n_positions", C.c_uint64), ("n_tokens", C.c_uint64),
                ("rot_dim", C.c_uint32), ("head_dim", C.c_uint32), ("dtype", C.c_uint32), ("weight_dtype", C.c_uint32),
                ("interleaved", C.c_uint32), ("eps", C.c_float)]


class _Attention(C.Structure):
    _fields_ = [("q", _Heads), ("out", _Heads), ("lse", C.c_void_p), ("k_pages", _Pages), ("v_pages", _Pages),
                ("group_offsets", C.c_void_p), ("prefix_tables", C.c_void_p), ("prefix_lens", C.c_void_p), ("q_offsets", C.c_void_p),
                ("own_tables", C.c_void_p), ("own_lens", C.c_void_p), ("n_tokens", C.c_uint64), ("n_requests", C.c_uint64),
                ("n_groups", C.c_uint64), ("prefix_width", C.c_uint64), ("own_width", C.c_uint64), ("n_pages", C.c_uint64),
                ("page_tokens", C.c_uint64), ("kv_heads", C.c_uint64), ("head_dim", C.c_uint32), ("dtype", C.c_uint32),
                ("scale", C.c_float), ("reserved", C.c_uint32)]


_lib = None


def _cache_lib():
    global _lib
    if _lib is None:
        L = _load()
        L.lsm_rope_table.restype = C.c_int
        L.lsm_rope_table.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32, C.c_double, C.c_void_p]
        L.lsm_rotate_heads.restype = C.c_int
        L.lsm_rotate_heads.argtypes = [C.POINTER(_Rotation), C.POINTER(_Heads), C.c_void_p, C.POINTER(_Heads), C.POINTER(_Heads), C.c_void_p,
                                       C.POINTER(_Heads), C.c_void_p]
        L.lsm_kv_append.restype = C.c_int
        L.lsm_kv_append.argtypes = [C.POINTER(_Rotation), C.POINTER(_Heads), C.c_void_p, C.POINTER(_Heads), C.c_void_p, C.POINTER(_Pages),
                                    C.POINTER(_Pages), C.c_uint64, C.c_uint64, C.POINTER(_Heads), C.c_void_p, C.POINTER(_Heads), C.c_void_p]
        L.lsm_prefix_attention_workspace_bytes.restype = C.c_size_t
        L.lsm_prefix_attention_workspace_bytes.argtypes = [C.POINTER(_Attention)]
        L.lsm_prefix_attention.restype = C.c_int
        L.lsm_prefix_attention.argtypes = [C.POINTER(_Attention), C.c_void_p, C.c_size_t, C.c_void_p]
        _lib = L
    return _lib


def _heads(t: torch.Tensor, what: str, tokens: int, head_dim: int, dtype: torch.dtype) -> _Heads:
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, is {t.dtype}")
    shape = t.shape
    if len(shape) != 3 or shape[0] != tokens or shape[2] != head_dim:
        raise ValueError(f"{what} must be [{tokens}, heads, {head_dim}], is {list(shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1:
        raise ValueError(f"{what}: the elements of a head must be contiguous")
    return _Heads(t.data_ptr(), s0, s1, shape[1])


def _pages(t: torch.Tensor, what: str, shape: Optional[torch.Size], dtype: torch.dtype) -> _Pages:
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, is {t.dtype}")
    if t.dim() != 4 or (shape is not None and t.shape != shape):
        raise ValueError(f"{what} must be [n_pages, page_tokens, kv_heads, head_dim]{'' if shape is None else f' = {list(shape)}'}, is {list(t.shape)}")
    s0, s1, s2, s3 = t.stride()
    if s3 != 1:
        raise ValueError(f"{what}: the elements of a head must be contiguous")
    return _Pages(t.data_ptr(), s0, s1, s2)


def _ints(t: torch.Tensor, what: str, shape: Tuple[int, ...], dtype: torch.dtype = torch.int32) -> int:
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} {list(shape)}, is {t.dtype} {list(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _rotation(x: torch.Tensor, positions, table, eps: float, interleaved: bool, weights) -> _Rotation:
    if x.dim() != 3:
        raise ValueError(f"heads must be [n_tokens, heads, head_dim], got {list(x.shape)}")
    dtype = _DTYPES.get(x.dtype)
    if dtype is None:
        raise ValueError(f"heads must be bfloat16, float16 or float32, got {x.dtype}")
    tokens, _, head_dim = x.shape
    weight_dtype = None
    for w in weights:
        if w is None:
            continue
        if not (w.is_cuda and w.is_contiguous() and w.shape == (head_dim,)):
            raise ValueError(f"a weight must be a contiguous GPU tensor of {head_dim} values")
        if w.dtype is not x.dtype and w.dtype is not torch.float32:
            raise ValueError(f"a weight must be {x.dtype} or float32, got {w.dtype}")
        if weight_dtype is not None and w.dtype is not weight_dtype:
            raise ValueError("the weights must have one type")
        weight_dtype = w.dtype
    r = _Rotation(0, 0, 0, tokens, 0, head_dim, dtype, dtype if weight_dtype is None else _DTYPES[weight_dtype], 1 if interleaved else 0, eps)
    if table is not None:
        if not (table.is_cuda and table.is_contiguous() and table.dtype is torch.float32 and table.dim() == 2):
            raise ValueError("the table must be a contiguous float32 GPU tensor [n_positions, rot_dim]")
        if positions is None:
            raise ValueError("a rotation needs positions")
        r.positions = _ints(positions, "positions", (tokens,))
        r.table = table.data_ptr()
        r.n_positions, r.rot_dim = table.shape
    return r


def lsm_rope_table(n_positions: int, rot_dim: int, theta: float = 10000.0, device="cuda", stream=None) -> torch.Tensor:
    """float32 [n_positions, rot_dim]: cosines, then sines, of the rotation's angles."""
    L = _cache_lib()
    table = torch.empty((n_positions, rot_dim), dtype=torch.float32, device=device)
    rc = L.lsm_rope_table(table.data_ptr(), n_positions, rot_dim, theta, _stream_ptr(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_rope_table")
    return table


def lsm_rotate_heads(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor], table: Optional[torch.Tensor], *,
                     q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     interleaved: bool = False, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(q_out, k_out): norm of every head (where there is a weight) and the position rotation (where there is a table).
    An output may be its input."""
    L = _cache_lib()
    x = q if q is not None else k
    if x is None:
        raise ValueError("lsm_rotate_heads needs q or k")
    how = _rotation(x, positions, table, eps, interleaved, (q_weight, k_weight))
    args = []
    outs = []
    for t, w, out, what in ((q, q_weight, q_out, "q"), (k, k_weight, k_out, "k")):
        if t is None:
            args += (None, None, None)
            outs.append(None)
            continue
        if out is None:
            out = torch.empty(t.shape, dtype=t.dtype, device=t.device)
        hi, ho = _heads(t, what, how.n_tokens, how.head_dim, x.dtype), _heads(out, what + "_out", how.n_tokens, how.head_dim, x.dtype)
        args += (C.byref(hi), w.data_ptr() if w is not None else None, C.byref(ho))
        outs.append(out)
    rc = L.lsm_rotate_heads(C.byref(how), *args, _stream_ptr(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_rotate_heads")
    return outs[0], outs[1]


def lsm_kv_append(k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor], slots: torch.Tensor, k_pages: torch.Tensor,
                  v_pages: torch.Tensor, table: Optional[torch.Tensor], *, k_weight: Optional[torch.Tensor] = None,
                  q: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                  eps: float = 1e-6, interleaved: bool = False, stream=None) -> Optional[torch.Tensor]:
    """Keys (normed, rotated) and values of the tokens into the slots of k_pages and v_pages; returns q normed and rotated
    if it is given."""
    L = _cache_lib()
    how = _rotation(k, positions, table, eps, interleaved, (q_weight, k_weight))
    tokens, head_dim, dtype = how.n_tokens, how.head_dim, k.dtype
    hk, hv = _heads(k, "k", tokens, head_dim, dtype), _heads(v, "v", tokens, head_dim, dtype)
    pk = _pages(k_pages, "k_pages", None, dtype)
    pv = _pages(v_pages, "v_pages", k_pages.shape, dtype)
    n_pages, page_tokens, kv_heads, d = k_pages.shape
    if kv_heads != hk.heads or kv_heads != hv.heads or d != head_dim:
        raise ValueError(f"k_pages must hold {hk.heads} heads of {head_dim}, has {kv_heads} of {d}")
    queries = (None, None, None)
    if q is not None:
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        hq, ho = _heads(q, "q", tokens, head_dim, dtype), _heads(q_out, "q_out", tokens, head_dim, dtype)
        queries = (C.byref(hq), q_weight.data_ptr() if q_weight is not None else None, C.byref(ho))
    rc = L.lsm_kv_append(C.byref(how), C.byref(hk), k_weight.data_ptr() if k_weight is not None else None, C.byref(hv),
                         _ints(slots, "slots", (tokens,), torch.int64), C.byref(pk), C.byref(pv), n_pages, page_tokens, *queries, _stream_ptr(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_kv_append")
    return q_out if q is not None else None


@dataclass
class PrefixBatch:
    """Which requests share which prefix, and where everybody's keys and values are (int32, see lsm_prefix_attention)."""
    group_offsets: torch.Tensor  # [n_groups + 1]               requests of each group
    prefix_tables: torch.Tensor  # [n_groups, prefix_width]     pages of each group's prefix
    prefix_lens: torch.Tensor    # [n_groups]                   its tokens
    q_offsets: torch.Tensor      # [n_requests + 1]             new tokens of each request
    own_tables: torch.Tensor     # [n_requests, own_width]      pages of each request's own tokens
    own_lens: torch.Tensor       # [n_requests]                 its own tokens, the new ones among them


def lsm_prefix_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, batch: PrefixBatch, *, scale: Optional[float] = None,
                         with_lse: bool = False, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of a batch whose requests share prefixes: out [n_tokens, heads, head_dim], or (out, lse [n_tokens, heads])."""
    L = _cache_lib()
    if q.dim() != 3:
        raise ValueError(f"q must be [n_tokens, heads, head_dim], is {list(q.shape)}")
    dtype = q.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise ValueError(f"q must be bfloat16 or float16, is {dtype}")
    tokens, heads, head_dim = q.shape
    if out is None:
        out = torch.empty(q.shape, dtype=dtype, device=q.device)
    lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if with_lse else None
    pk = _pages(k_pages, "k_pages", None, dtype)
    pv = _pages(v_pages, "v_pages", k_pages.shape, dtype)
    n_pages, page_tokens, kv_heads, d = k_pages.shape
    if d != head_dim:
        raise ValueError(f"k_pages must hold heads of {head_dim}, has {d}")
    if batch.prefix_tables.dim() != 2 or batch.own_tables.dim() != 2:
        raise ValueError("prefix_tables and own_tables must be [groups, pages] and [requests, pages]")
    n_groups, prefix_width = batch.prefix_tables.shape
    n_requests, own_width = batch.own_tables.shape
    a = _Attention(_heads(q, "q", tokens, head_dim, dtype), _heads(out, "out", tokens, head_dim, dtype), lse.data_ptr() if with_lse else None, pk, pv,
                   _ints(batch.group_offsets, "group_offsets", (n_groups + 1,)), _ints(batch.prefix_tables, "prefix_tables", (n_groups, prefix_width)),
                   _ints(batch.prefix_lens, "prefix_lens", (n_groups,)), _ints(batch.q_offsets, "q_offsets", (n_requests + 1,)),
                   _ints(batch.own_tables, "own_tables", (n_requests, own_width)), _ints(batch.own_lens, "own_lens", (n_requests,)),
                   tokens, n_requests, n_groups, prefix_width, own_width, n_pages, page_tokens, kv_heads, head_dim, _DTYPES[dtype],
                   head_dim ** -0.5 if scale is None else scale, 0)
    ref = C.byref(a)
    if workspace is None:
        need = L.lsm_prefix_attention_workspace_bytes(ref)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    rc = L.lsm_prefix_attention(ref, workspace.data_ptr() if workspace is not None else None, workspace.numel() if workspace is not None else 0,
                                _stream_ptr(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_prefix_attention")
    return (out, lse) if with_lse else out
