"""Binding of the paged 16-bit cache (cocktail_kv16_*): pages of K and V in float16 or bfloat16 on the page tables of `paged`, with the
position rotation on the way into them.  Streams, workspaces and threads as there.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from . import _lib
from ._lib import check, lib
from .paged import _DTYPES, PageTable, _here, _on, _rows, _starts, _used_on


class Kv16Cache:
    """One layer's pools of K and V in 16 bits, [num_pages, num_kv_heads, page_size, head_dim] each, addressed by a page table that layers share.
    `pools` (what cocktail_pages_resize and cocktail_pages_compact take) is (k, v)."""

    def __init__(self, pages: PageTable, num_kv_heads: int, head_dim: int, dtype: torch.dtype = torch.float16,
                 pools: Optional[Tuple[torch.Tensor, torch.Tensor]] = None):
        if dtype not in _DTYPES:
            raise TypeError("dtype must be float16 or bfloat16")
        shape = (pages.num_pages, int(num_kv_heads), pages.page_size, int(head_dim))
        if pools is None:
            pools = tuple(torch.empty(shape, dtype=dtype, device=pages.device) for _ in range(2))
        for t in pools:
            if t.dtype != dtype or t.device != pages.device or not t.is_contiguous() or tuple(t.shape) != shape:
                raise TypeError(f"the pools must be contiguous {dtype} tensors {list(shape)} on {pages.device}")
        self.k, self.v = pools
        if abs(self.k.data_ptr() - self.v.data_ptr()) < self.k.nbytes:
            raise ValueError("K and V must have pools of their own")
        self.pages, self.pools, self.dtype = pages, (self.k, self.v), dtype
        self.num_kv_heads, self.head_dim = int(num_kv_heads), int(head_dim)
        self.desc = _lib.Kv16CacheDesc(pages.desc, self.k.data_ptr(), self.v.data_ptr(), self.num_kv_heads, self.head_dim, _DTYPES[dtype], 0)
        self.desc_ref = C.byref(self.desc)
        need = C.c_size_t(0)
        check(lib().cocktail_kv16_attention_workspace(self.desc_ref, self.num_kv_heads, 0, 0, 0, 0, C.byref(need)))   # checks the sizes
        self.workspace_bytes = {}   # by the sizes of the call


class Rotation:
    """Rotation of pairs of channels by the position: pair i turns by position * inv_freq[i].  inv_freq: float64 [rotary_dim / 2] on the device; pairs are
    channels i and i + rotary_dim / 2, or neighbours if `interleaved`; `factor` multiplies the result."""

    def __init__(self, inv_freq: torch.Tensor, interleaved: bool = False, factor: float = 1.0):
        if not inv_freq.is_cuda or inv_freq.dtype != torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise TypeError("inv_freq must be a contiguous float64 device tensor [rotary_dim / 2]")
        self.inv_freq, self.device = inv_freq, inv_freq.device
        self.desc = _lib.RotationDesc(inv_freq.data_ptr(), 2 * inv_freq.numel(), 1 if interleaved else 0, float(factor), 0)
        self.desc_ref = C.byref(self.desc)


def _of_cache(name: str, t: torch.Tensor, cache: Kv16Cache, heads: int) -> Tuple[int, int, int]:
    if t.dtype != cache.dtype:
        raise TypeError(f"{name} must have the cache's type, {cache.dtype}")
    return _rows(name, t, heads, cache.head_dim, cache.pages.device)


def cocktail_kv16_append(cache: Kv16Cache, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None,
                         rotation: Optional[Rotation] = None, q: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                         q_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> Optional[torch.Tensor]:
    """Appends new tokens: rows starts[b] .. starts[b+1] of k and v ([tokens, Hkv, D]) become the last tokens of sequence b, k rotated by `rotation`.
    Without `starts` every sequence has the same number of rows.  Call cocktail_pages_resize first: it makes the room.  q [tokens, Hq, D], the queries of
    the same tokens, are rotated into q_out, which is returned (q itself, if contiguous, or a new tensor).  positions: device int32 [tokens] for
    the rotation (default: the tokens' numbers in their sequences)."""
    dev = cache.pages.device
    handle = _here(dev, stream)
    if handle is None:
        with _on(dev, stream):
            result = cocktail_kv16_append(cache, k, v, starts, rotation, q, positions, q_out)
        _used_on(stream, cache.pages, cache.k, cache.v, k, v, starts, q, positions, result, rotation.inv_freq if rotation else None)
        return result
    rows = _of_cache("k", k, cache, cache.num_kv_heads)
    if rows != _of_cache("v", v, cache, cache.num_kv_heads):
        raise ValueError("k and v must have the same shape and strides")
    if rotation is not None and rotation.device != dev:
        raise TypeError(f"inv_freq must be on {dev}")
    at = None
    if positions is not None:
        if positions.dtype != torch.int32 or positions.device != dev or tuple(positions.shape) != (rows[0],) or not positions.is_contiguous():
            raise TypeError(f"positions must be a contiguous int32 tensor [{rows[0]}] on {dev}")
        at = positions.data_ptr()
    heads, st, sh, src, dst = 0, 0, 0, None, None
    if q is not None:
        if q.dim() != 3:
            raise TypeError("q must be [tokens, Hq, D]")
        heads = q.shape[1]
        total, st, sh = _of_cache("q", q, cache, heads)
        if total != rows[0]:
            raise ValueError("q must have as many rows as k and v")
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif q_out.dtype != q.dtype or q_out.shape != q.shape or q_out.device != dev or not q_out.is_contiguous():
            raise ValueError("q_out must be a contiguous tensor of q's type, shape and device")
        if total == 0:
            heads = 0   # (no rows have no address)
        else:
            src, dst = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out is for q")
    check(lib().cocktail_kv16_append(cache.desc_ref, k.data_ptr(), v.data_ptr(), rows[1], rows[2], rows[0], _starts(cache, starts),
                                     rotation.desc_ref if rotation is not None else None, at, src, heads, st, sh, dst, handle))
    return q_out


def cocktail_kv16_attention(cache: Kv16Cache, q: torch.Tensor, starts: Optional[torch.Tensor] = None, max_new: Optional[int] = None,
                            max_len: int = 0, sm_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                            lse: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Causal attention of the newest tokens of every sequence, q [tokens, Hq, D] of the cache's type, over the cached keys, themselves included.
    Returns (out, lse).  max_new: no sequence has more queries (default: as many as there are rows); max_len: about the longest
    sequence, for the split of the work (default: what the table can hold)."""
    dev = cache.pages.device
    handle = _here(dev, stream)
    if handle is None:
        with _on(dev, stream):
            result = cocktail_kv16_attention(cache, q, starts, max_new, max_len, sm_scale, out, lse)
        _used_on(stream, cache.pages, cache.k, cache.v, q, starts, out, lse)
        return result
    if q.dim() != 3:
        raise TypeError("q must be [tokens, Hq, D]")
    heads = q.shape[1]
    total, st, sh = _of_cache("q", q, cache, heads)
    if max_new is None:
        max_new = total // cache.pages.num_seqs if starts is None else total
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.dtype != q.dtype or out.shape != q.shape or out.device != dev or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of q's type, shape and device")
    if lse is None:
        lse = torch.empty_strided((total, heads), (heads, 1), dtype=torch.float32, device=dev)
    elif lse.dtype != torch.float32 or tuple(lse.shape) != (total, heads) or lse.device != dev or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 tensor [tokens, Hq]")
    first = _starts(cache, starts)
    key = (heads, total, max_new, max_len, starts is None)
    need = cache.workspace_bytes.get(key)
    if need is None:
        size = C.c_size_t(0)
        check(lib().cocktail_kv16_attention_workspace(cache.desc_ref, heads, total, int(max_new), int(max_len), 1 if starts is None else 0,
                                                      C.byref(size)))
        if len(cache.workspace_bytes) > 4096:
            cache.workspace_bytes.clear()
        need = cache.workspace_bytes[key] = int(size.value)
    workspaces = cache.pages.workspaces
    with workspaces.lock:
        workspace = workspaces.get(need, handle)
        check(lib().cocktail_kv16_attention(cache.desc_ref, heads, q.data_ptr(), st, sh, total, first, int(max_new), int(max_len), float(sm_scale),
                                            out.data_ptr(), lse.data_ptr(), workspace.data_ptr(), need, handle))
    return out, lse
