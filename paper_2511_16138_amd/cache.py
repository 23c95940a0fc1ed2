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
import struct
from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from .binding import LsmError, _load, _stream_ptr

_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}

# The descriptors of lsm_cache.h as packed bytes: a call of a few microseconds on the GPU should not wait for ctypes structures.
_HEADS = struct.Struct("=QqqQ")                  # lsm_heads_t
_PAGES = struct.Struct("=Qqqq")                  # lsm_pages_t
_ROTATION = struct.Struct("=4Q5If")              # lsm_rotation_t
_ATTENTION = struct.Struct("=QqqQQqqQQQqqqQqqq6Q8QIIfI")  # lsm_attention_t

_lib = None


def _cache_lib():
    global _lib
    if _lib is None:
        L = _load()
        b, p, n = C.c_char_p, C.c_void_p, C.c_uint64
        L.lsm_rope_table.restype = C.c_int
        L.lsm_rope_table.argtypes = [p, n, C.c_uint32, C.c_double, p]
        L.lsm_rotate_heads.restype = C.c_int
        L.lsm_rotate_heads.argtypes = [b, b, p, b, b, p, b, p]
        L.lsm_kv_append.restype = C.c_int
        L.lsm_kv_append.argtypes = [b, b, p, b, p, b, b, n, n, b, p, b, p]
        L.lsm_prefix_attention_workspace_bytes.restype = C.c_size_t
        L.lsm_prefix_attention_workspace_bytes.argtypes = [b]
        L.lsm_prefix_attention.restype = C.c_int
        L.lsm_prefix_attention.argtypes = [b, p, C.c_size_t, p]
        _lib = L
    return _lib


def _heads(t: torch.Tensor, what: str, tokens: int, head_dim: int, dtype: torch.dtype) -> Tuple[int, int, int, int]:
    """lsm_heads_t of [tokens, heads, head_dim]."""
    shape, strides = t.shape, t.stride()
    if t.is_cuda and t.dtype is dtype and len(shape) == 3 and shape[0] == tokens and shape[2] == head_dim and strides[2] == 1:
        return t.data_ptr(), strides[0], strides[1], shape[1]
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if t.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype}, is {t.dtype}")
    if len(shape) != 3 or shape[0] != tokens or shape[2] != head_dim:
        raise ValueError(f"{what} must be [{tokens}, heads, {head_dim}], is {list(shape)}")
    raise ValueError(f"{what}: the elements of a head must be contiguous")


def _pages(t: torch.Tensor, what: str, shape, dtype: torch.dtype) -> Tuple[int, int, int, int]:
    """lsm_pages_t of [n_pages, page_tokens, kv_heads, head_dim]."""
    strides = t.stride()
    if t.is_cuda and t.dtype is dtype and len(strides) == 4 and t.shape == shape and strides[3] == 1:
        return t.data_ptr(), strides[0], strides[1], strides[2]
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if t.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype}, is {t.dtype}")
    if len(strides) != 4 or t.shape != shape:
        raise ValueError(f"{what} must be [n_pages, page_tokens, kv_heads, head_dim] as k_pages is {list(shape)}, is {list(t.shape)}")
    raise ValueError(f"{what}: the elements of a head must be contiguous")


def _ints(t: torch.Tensor, what: str, shape: Tuple[int, ...], dtype: torch.dtype = torch.int32) -> int:
    if t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} {list(shape)}, is {t.dtype} {list(t.shape)}")
    raise ValueError(f"{what} must be contiguous")


def _new_like(t: torch.Tensor, stream) -> torch.Tensor:
    return _used_on(torch.empty_like(t, memory_format=torch.contiguous_format), stream)


def _used_on(t: torch.Tensor, stream) -> torch.Tensor:
    """A tensor made here (on torch's current stream) that work on `stream`, a caller's own, is going to use."""
    if stream is not None:
        t.record_stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=t.device))
    return t


def _rotation(x: torch.Tensor, positions, table, eps: float, interleaved: bool, w0, w1) -> bytes:
    dtype = x.dtype
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"heads must be bfloat16, float16 or float32, got {dtype}")
    if x.dim() != 3:
        raise ValueError(f"heads must be [n_tokens, heads, head_dim], got {list(x.shape)}")
    tokens, _, head_dim = x.shape
    weight_dtype = dtype
    if w0 is not None or w1 is not None:
        weight_dtype = (w1 if w0 is None else w0).dtype
        if weight_dtype is not dtype and weight_dtype is not torch.float32:
            raise ValueError(f"a weight must be {dtype} or float32, got {weight_dtype}")
        for w in (w0, w1):
            if w is not None and not (w.is_cuda and w.dtype is weight_dtype and w.shape == (head_dim,) and w.is_contiguous()):
                raise ValueError(f"the weights must be contiguous GPU tensors of {head_dim} values of one type")
    if table is None:
        return _ROTATION.pack(0, 0, 0, tokens, 0, head_dim, code, _DTYPES[weight_dtype], 1 if interleaved else 0, eps)
    if not (table.is_cuda and table.dtype is torch.float32 and table.dim() == 2 and table.is_contiguous()):
        raise ValueError("the table must be a contiguous float32 GPU tensor [n_positions, rot_dim]")
    if positions is None:
        raise ValueError("a rotation needs positions")
    n_positions, rot_dim = table.shape
    return _ROTATION.pack(_ints(positions, "positions", (tokens,)), table.data_ptr(), n_positions, tokens, rot_dim, head_dim, code,
                          _DTYPES[weight_dtype], 1 if interleaved else 0, eps)


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
    x = q if q is not None else k
    if x is None:
        raise ValueError("lsm_rotate_heads needs q or k")
    L = _cache_lib()
    how = _rotation(x, positions, table, eps, interleaved, q_weight, k_weight)
    tokens, _, head_dim = x.shape
    dtype = x.dtype
    qi = qo = wq = ki = ko = wk = None
    if q is not None:
        if q_out is None:
            q_out = _new_like(q, stream)
        qi, qo = _HEADS.pack(*_heads(q, "q", tokens, head_dim, dtype)), _HEADS.pack(*_heads(q_out, "q_out", tokens, head_dim, dtype))
        wq = None if q_weight is None else q_weight.data_ptr()
    if k is not None:
        if k_out is None:
            k_out = _new_like(k, stream)
        ki, ko = _HEADS.pack(*_heads(k, "k", tokens, head_dim, dtype)), _HEADS.pack(*_heads(k_out, "k_out", tokens, head_dim, dtype))
        wk = None if k_weight is None else k_weight.data_ptr()
    rc = L.lsm_rotate_heads(how, qi, wq, qo, ki, wk, ko, _stream_ptr(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_rotate_heads")
    return (q_out if q is not None else None), (k_out if k is not None else None)


def lsm_kv_append(k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor], slots: torch.Tensor, k_pages: torch.Tensor,
                  v_pages: torch.Tensor, table: Optional[torch.Tensor], *, k_weight: Optional[torch.Tensor] = None,
                  q: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                  eps: float = 1e-6, interleaved: bool = False, stream=None) -> Optional[torch.Tensor]:
    """Keys (normed, rotated) and values of the tokens into the slots of k_pages and v_pages; returns q normed and rotated
    if it is given."""
    L = _cache_lib()
    how = _rotation(k, positions, table, eps, interleaved, q_weight, k_weight)
    tokens, heads, head_dim = k.shape
    dtype, shape = k.dtype, k_pages.shape
    if len(shape) != 4 or shape[2] != heads or shape[3] != head_dim or v.size(1) != heads:
        raise ValueError(f"k_pages must be [n_pages, page_tokens, {heads}, {head_dim}] and v have {heads} heads, are {list(shape)} and {list(v.shape)}")
    qi = qo = wq = None
    if q is not None:
        if q_out is None:
            q_out = _new_like(q, stream)
        qi, qo = _HEADS.pack(*_heads(q, "q", tokens, head_dim, dtype)), _HEADS.pack(*_heads(q_out, "q_out", tokens, head_dim, dtype))
        wq = None if q_weight is None else q_weight.data_ptr()
    rc = L.lsm_kv_append(how, _HEADS.pack(*_heads(k, "k", tokens, head_dim, dtype)), None if k_weight is None else k_weight.data_ptr(),
                         _HEADS.pack(*_heads(v, "v", tokens, head_dim, dtype)), _ints(slots, "slots", (tokens,), torch.int64),
                         _PAGES.pack(*_pages(k_pages, "k_pages", shape, dtype)), _PAGES.pack(*_pages(v_pages, "v_pages", shape, dtype)),
                         shape[0], shape[1], qi, wq, qo, _stream_ptr(stream))
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
    dtype, q_shape, shape = q.dtype, q.shape, k_pages.shape
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise ValueError(f"q must be bfloat16 or float16, is {dtype}")
    if len(q_shape) != 3 or len(shape) != 4 or q_shape[2] != shape[3]:
        raise ValueError(f"q and k_pages must be [n_tokens, heads, head_dim] and [n_pages, page_tokens, kv_heads, head_dim], are {list(q_shape)} and {list(shape)}")
    tokens, heads, head_dim = q_shape
    prefix_tables, own_tables = batch.prefix_tables, batch.own_tables
    if prefix_tables.dim() != 2 or own_tables.dim() != 2:
        raise ValueError("prefix_tables and own_tables must be [n_groups, prefix_width] and [n_requests, own_width]")
    n_groups, prefix_width = prefix_tables.shape
    n_requests, own_width = own_tables.shape
    if out is None:
        out = _new_like(q, stream)
    lse = _used_on(torch.empty((tokens, heads), dtype=torch.float32, device=q.device), stream) if with_lse else None
    a = _ATTENTION.pack(*_heads(q, "q", tokens, head_dim, dtype), *_heads(out, "out", tokens, head_dim, dtype), lse.data_ptr() if with_lse else 0,
                        *_pages(k_pages, "k_pages", shape, dtype), *_pages(v_pages, "v_pages", shape, dtype),
                        _ints(batch.group_offsets, "group_offsets", (n_groups + 1,)), _ints(prefix_tables, "prefix_tables", (n_groups, prefix_width)),
                        _ints(batch.prefix_lens, "prefix_lens", (n_groups,)), _ints(batch.q_offsets, "q_offsets", (n_requests + 1,)),
                        _ints(own_tables, "own_tables", (n_requests, own_width)), _ints(batch.own_lens, "own_lens", (n_requests,)),
                        tokens, n_requests, n_groups, prefix_width, own_width, shape[0], shape[1], shape[2], head_dim, _DTYPES[dtype],
                        head_dim ** -0.5 if scale is None else scale, 0)
    if workspace is None:
        need = L.lsm_prefix_attention_workspace_bytes(a)
        if need:
            workspace = _used_on(torch.empty(need, dtype=torch.uint8, device=q.device), stream)
    elif not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous GPU tensor")
    rc = L.lsm_prefix_attention(a, None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                _stream_ptr(stream))
    if rc != 0:
        raise LsmError(rc, "lsm_prefix_attention")
    return (out, lse) if with_lse else out


def lsm_prefix_attention_workspace_bytes(n_tokens: int, heads: int, head_dim: int, kv_heads: int, n_requests: int, n_groups: int, prefix_width: int,
                                         own_width: int, page_tokens: int, dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of workspace that lsm_prefix_attention needs for these sizes (the ones of its tensors' shapes)."""
    one = 256  # no address is used
    a = _ATTENTION.pack(one, 0, 0, heads, one, 0, 0, heads, 0, one, 0, 0, 0, one, 0, 0, 0, one, one, one, one, one, one, n_tokens, n_requests, n_groups,
                        prefix_width, own_width, 1, page_tokens, kv_heads, head_dim, _DTYPES[dtype], 1.0, 0)
    return int(_cache_lib().lsm_prefix_attention_workspace_bytes(a))
