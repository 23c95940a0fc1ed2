"""The paged-cache calls of liblsm_index.so (include/lsm_cache.h; same names as the C entry points) on torch tensors.

Tensors are on the current GPU:
  q, k, v          [n_tokens, heads, head_dim], any strides with contiguous elements of a head; bfloat16, float16 (or float32,
                   not for attention)
  k_pages, v_pages [n_pages, page_tokens, kv_heads, head_dim], any strides likewise: a layer's slice of blocks that hold all
                   layers' keys and values is fine
  positions, page tables, lengths, offsets   int32, contiguous;  slots   int64, contiguous

Work goes to torch's current stream, or to `stream` (a torch stream or a HIP stream handle), which is then the current one while
outputs and workspace are made.  Wrong shapes and types raise ValueError, errors of the library LsmError; nothing is launched then.
There is no backward pass and no forward mode: an input or output that requires gradients (where torch's grad mode is on) or has a tangent raises ValueError.
The marshalling is compiled (csrc/lsm_cache_torch.cpp); there is no fallback: a missing module raises at the first call.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import Optional, Tuple

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
                         with_lse: bool = False, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of a batch whose requests share prefixes: out [n_tokens, heads, head_dim], or (out, lse [n_tokens, heads])."""
    call = (_calls or _module()).prefix_attention
    b = batch
    if stream is None:
        r = call(q, k_pages, v_pages, b.group_offsets, b.prefix_tables, b.prefix_lens, b.q_offsets, b.own_tables, b.own_lens, scale, with_lse, out, workspace)
    else:
        r = _on(stream, call, q, k_pages, v_pages, b.group_offsets, b.prefix_tables, b.prefix_lens, b.q_offsets, b.own_tables, b.own_lens, scale, with_lse,
                out, workspace)
    if type(r) is int:
        raise LsmError(r, "lsm_prefix_attention")
    return r
