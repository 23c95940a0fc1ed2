"""The paged-cache calls of liblsm_index.so (include/lsm_cache.h, include/lsm_pages.h; same names as the C entry points) on torch tensors.

Tensors are on the current GPU:
  q, k, v          [n_tokens, heads, head_dim], any strides with contiguous elements of a head; bfloat16, float16 (or float32,
                   not for attention)
  k_pages, v_pages [n_pages, page_tokens, kv_heads, head_dim], any strides likewise: a layer's slice of blocks that hold all
                   layers' keys and values is fine
                   in 8 bits: float8_e4m3fn, with
  k_scales, v_scales float8_e8m0fnu [n_pages, page_tokens / 16, kv_heads], any strides: a value is code * scale, one scale for 16 tokens of a head
  positions, page tables, lengths, offsets   int32, contiguous;  slots   int64, contiguous

Work goes to torch's current stream, or to `stream` (a torch stream or a HIP stream handle), which is then the current one while
outputs and workspace are made.  Wrong shapes and types raise ValueError, errors of the library LsmError; nothing is launched then.
There is no backward pass and no forward mode: an input or output that requires gradients (where torch's grad mode is on) or has a tangent raises ValueError.
The marshalling is compiled (csrc/lsm_cache_torch.cpp); there is no fallback: a missing module raises at the first call.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import List, Optional, Sequence, Tuple, Union

import torch

from .binding import LsmError, _load, _stream_ptr

_calls = None


def _module():
    global _calls
    if _calls is None:
        try:
            from . import _cache
        except ImportError as e:
            raise RuntimeError(f"paper_2511_16138_amd/_cache.so cannot be loaded ({e}): build it first (__graft_entry__.build()); there is no fallback") from e
        _calls = _cache
    return _calls


def _on(stream, call, *args):
    """call(*args) with `stream` as torch's current stream."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream))
    with torch.cuda.stream(stream):
        return call(*args)


def lsm_rope_table(n_positions: int, rot_dim: int, theta: float = 10000.0, device="cuda", stream=None) -> torch.Tensor:
    """float32 [n_positions, rot_dim]: cosines, then sines, of the rotation's angles.  device: the current GPU ("cuda", or its own number)."""
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError(f"device must be the current GPU, is {device}")
    L = _load()
    if not hasattr(L.lsm_rope_table, "typed"):
        L.lsm_rope_table.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32, C.c_double, C.c_void_p]
        L.lsm_rope_table.typed = True
    if n_positions < 0 or rot_dim <= 0:
        raise ValueError("n_positions must not be negative and rot_dim be above 0")
    if stream is not None:
        return _on(stream, lsm_rope_table, n_positions, rot_dim, theta, device)
    if device.index not in (None, torch.cuda.current_device()):
        raise ValueError(f"device must be the current GPU ({torch.cuda.current_device()}), is {device}")
    table = torch.empty((n_positions, rot_dim), dtype=torch.float32, device=device)
    rc = L.lsm_rope_table(table.data_ptr(), n_positions, rot_dim, theta, _stream_ptr(None))
    if rc != 0:
        raise LsmError(rc, "lsm_rope_table")
    return table


def lsm_rotate_heads(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor], table: Optional[torch.Tensor], *,
                     q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     interleaved: bool = False, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(q_out, k_out): norm of every head (where there is a weight) and the position rotation (where there is a table).
    An output may be its input."""
    call = (_calls or _module()).rotate_heads
    if stream is None:
        r = call(q, k, positions, table, q_weight, k_weight, eps, interleaved, q_out, k_out)
    else:
        r = _on(stream, call, q, k, positions, table, q_weight, k_weight, eps, interleaved, q_out, k_out)
    if type(r) is int:
        raise LsmError(r, "lsm_rotate_heads")
    return r


def lsm_kv_append(k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor], slots: torch.Tensor, k_pages: torch.Tensor,
                  v_pages: torch.Tensor, table: Optional[torch.Tensor], *, k_weight: Optional[torch.Tensor] = None,
                  q: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                  eps: float = 1e-6, interleaved: bool = False, stream=None) -> Optional[torch.Tensor]:
    """Keys (normed, rotated) and values of the tokens into the slots of k_pages and v_pages; returns q normed and rotated
    if it is given."""
    call = (_calls or _module()).kv_append
    if stream is None:
        r = call(k, v, positions, slots, k_pages, v_pages, table, k_weight, q, q_weight, q_out, eps, interleaved)
    else:
        r = _on(stream, call, k, v, positions, slots, k_pages, v_pages, table, k_weight, q, q_weight, q_out, eps, interleaved)
    if type(r) is int:
        raise LsmError(r, "lsm_kv_append")
    return r


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
                         with_lse: bool = False, k_scales: Optional[torch.Tensor] = None, v_scales: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0,
                         out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of a batch whose requests share prefixes: out [n_tokens, heads, head_dim], or (out, lse [n_tokens, heads]).

    k_scales, v_scales: the pages are in 8 bits.  window: a token sees the last `window` tokens of its sequence (prefix, then own), itself among them, and
    the first `sinks`; 0: all of them.  (lsm_window_attention of the C library, where any of these is given.)"""
    more = k_scales is not None or v_scales is not None or window != 0 or sinks != 0
    call = (_calls or _module()).window_attention if more else (_calls or _module()).prefix_attention
    b = batch
    args = (q, k_pages, v_pages, b.group_offsets, b.prefix_tables, b.prefix_lens, b.q_offsets, b.own_tables, b.own_lens, scale, with_lse, out, workspace)
    if more:
        args += (k_scales, v_scales, window, sinks)
    r = call(*args) if stream is None else _on(stream, call, *args)
    if type(r) is int:
        raise LsmError(r, "lsm_window_attention" if more else "lsm_prefix_attention")
    return r


def lsm_kv_append8(k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor], batch: PrefixBatch, k_pages: torch.Tensor, v_pages: torch.Tensor,
                   k_scales: torch.Tensor, v_scales: torch.Tensor, table: Optional[torch.Tensor], *, k_weight: Optional[torch.Tensor] = None,
                   q: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                   eps: float = 1e-6, interleaved: bool = False, stream=None) -> Optional[torch.Tensor]:
    """Keys (normed, rotated) and values of the batch's new tokens into pages of 8 bits, where lsm_prefix_attention looks for them; returns q normed and
    rotated if it is given.  Of the batch, q_offsets, own_tables and own_lens count."""
    call = (_calls or _module()).kv_append8
    b = batch
    args = (k, v, positions, b.q_offsets, b.own_tables, b.own_lens, k_pages, v_pages, k_scales, v_scales, table, k_weight, q, q_weight, q_out, eps, interleaved)
    r = call(*args) if stream is None else _on(stream, call, *args)
    if type(r) is int:
        raise LsmError(r, "lsm_kv_append8")
    return r


def lsm_copy_pages(pages: Union[torch.Tensor, Sequence[torch.Tensor]], sources: torch.Tensor, targets: torch.Tensor, *, stream=None) -> None:
    """Page targets[i] becomes a copy of page sources[i] in every tensor [n_pages, ...] of any type whose pages are single stretches of memory."""
    call = (_calls or _module()).copy_pages
    r = call(pages, sources, targets) if stream is None else _on(stream, call, pages, sources, targets)
    if type(r) is int:
        raise LsmError(r, "lsm_copy_pages")


def lsm_compact_pages(pages: Union[torch.Tensor, Sequence[torch.Tensor]], tables: Union[torch.Tensor, Sequence[torch.Tensor]],
                      lens: Union[torch.Tensor, Sequence[torch.Tensor]], page_tokens: int, *, n_pages: Optional[int] = None,
                      stream=None) -> Tuple[List[torch.Tensor], torch.Tensor, torch.Tensor]:
    """Moves the pages that the tables hold together: (new tables, moved [n_pages], n_live [1]).  Entry j of a row of a table [rows, width] holds a page if
    j * page_tokens < lens[row]; moved is a page's new number, -1 for a free one; pages from n_live on are free afterwards.  pages: as for lsm_copy_pages, or [] with
    n_pages given, for the plan alone."""
    call = (_calls or _module()).compact_pages
    args = (pages, tables, lens, page_tokens, n_pages)
    r = call(*args) if stream is None else _on(stream, call, *args)
    if type(r) is int:
        raise LsmError(r, "lsm_compact_pages")
    new_tables, (moved, n_live) = r
    return new_tables, moved, n_live
