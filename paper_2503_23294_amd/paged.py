"""Binding of the paged 4-bit cache: the page table (cocktail_pages_*) and the cache on top of it (cocktail_fp4_*).

Same names as the C entry points.  torch supplies device memory and streams; workspaces are taken from its allocator per call, in the
order of the call's stream, so that calls on several streams or in several captured graphs never share one.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Sequence, Tuple

import torch

from . import _lib
from ._lib import check, lib
from .api import _stream_ptr

_DTYPES = {torch.float16: _lib.FP16, torch.bfloat16: _lib.BF16}


def _on(device: torch.device, stream: Optional[torch.cuda.Stream]):
    """Makes the tensors' device current for the call, and the stream for what is allocated in it."""
    if stream is not None:
        if stream.device != device:
            raise ValueError("the stream belongs to another device than the tensors")
        return torch.cuda.stream(stream)
    if device.index != torch.cuda.current_device():
        return torch.cuda.device(device)
    return contextlib.nullcontext()


def _int32(name: str, t: torch.Tensor, shape: Tuple[int, ...], device: torch.device) -> None:
    if t.dtype != torch.int32 or t.device != device or not t.is_contiguous() or tuple(t.shape) != shape:
        raise TypeError(f"{name} must be a contiguous int32 tensor {list(shape)} on {device}")


class PageTable:
    """Which pages the sequences of a batch have, how long they are, and how many table entries name each page (all on the device)."""

    def __init__(self, num_seqs: int, max_tokens: int, num_pages: int, page_size: int, device: torch.device):
        device = torch.device(device)
        columns = -(-int(max_tokens) // int(page_size))
        self._set(torch.full((num_seqs, columns), -1, dtype=torch.int32, device=device),
                  torch.zeros(num_seqs, dtype=torch.int32, device=device),
                  torch.zeros(num_pages, dtype=torch.int32, device=device), int(page_size), None)

    @classmethod
    def of(cls, table: torch.Tensor, seq_lens: torch.Tensor, refs: torch.Tensor, page_size: int,
           status: Optional[torch.Tensor] = None) -> "PageTable":
        """A page table in tensors that are there already: table [num_seqs, pages per sequence], seq_lens [num_seqs], refs [num_pages]."""
        self = cls.__new__(cls)
        self._set(table, seq_lens, refs, int(page_size), status)
        return self

    def _set(self, table, seq_lens, refs, page_size, status):
        if not table.is_cuda or table.dim() != 2:
            raise TypeError("table must be a device tensor [num_seqs, pages per sequence]")
        dev = table.device
        _int32("table", table, tuple(table.shape), dev)
        _int32("seq_lens", seq_lens, (table.shape[0],), dev)
        _int32("refs", refs, (refs.numel(),), dev)
        if status is None:
            status = torch.zeros(4, dtype=torch.int32, device=dev)
        _int32("status", status, (4,), dev)
        self.table, self.seq_lens, self.refs, self.status = table, seq_lens, refs, status
        self.page_size, self.device = page_size, dev
        self.desc = _lib.PageTableDesc(table.data_ptr(), seq_lens.data_ptr(), refs.data_ptr(), status.data_ptr(), table.shape[0],
                                       table.shape[1], page_size, refs.shape[0])
        need = C.c_size_t(0)
        check(lib().cocktail_pages_workspace(C.byref(self.desc), C.byref(need)))   # also checks the sizes
        self.workspace_bytes = int(need.value)

    @property
    def num_seqs(self) -> int:
        return int(self.table.shape[0])

    @property
    def num_pages(self) -> int:
        return int(self.refs.shape[0])


class Fp4Cache:
    """One layer's pool of pages in microscaled 4-bit floating point, addressed by a page table that layers share."""

    def __init__(self, pages: PageTable, num_kv_heads: int, head_dim: int, pool: Optional[torch.Tensor] = None):
        need = C.c_int64(0)
        check(lib().cocktail_fp4_page_bytes(int(num_kv_heads), int(head_dim), pages.page_size, C.byref(need)))
        self.page_bytes = int(need.value)
        if pool is None:
            pool = torch.empty(pages.num_pages, self.page_bytes, dtype=torch.uint8, device=pages.device)
        if pool.dtype != torch.uint8 or pool.device != pages.device or not pool.is_contiguous() or \
                tuple(pool.shape) != (pages.num_pages, self.page_bytes):
            raise TypeError(f"pool must be a contiguous uint8 tensor [{pages.num_pages}, {self.page_bytes}] on {pages.device}")
        self.pages, self.pool = pages, pool
        self.num_kv_heads, self.head_dim = int(num_kv_heads), int(head_dim)
        self.desc = _lib.Fp4CacheDesc(pages.desc, pool.data_ptr(), self.num_kv_heads, self.head_dim)


def _pool_list(pages: PageTable, pools: Sequence[torch.Tensor]):
    """ctypes array of the pools' addresses, their number and the bytes of a page."""
    bytes_per_page = 0
    array = (C.c_void_p * max(1, len(pools)))()
    for i, t in enumerate(pools):
        if t.device != pages.device or not t.is_contiguous() or t.dim() < 1 or t.shape[0] != pages.num_pages:
            raise TypeError(f"pools must be contiguous tensors [{pages.num_pages}, ...] on {pages.device}")
        n = t.numel() // pages.num_pages * t.element_size()
        if i and n != bytes_per_page:
            raise ValueError("the pools of a call must have pages of the same size")
        bytes_per_page = n
        array[i] = t.data_ptr()
    return array, len(pools), bytes_per_page


def cocktail_pages_resize(pages: PageTable, delta: torch.Tensor, pools: Sequence[torch.Tensor] = (),
                          stream: Optional[torch.cuda.Stream] = None) -> None:
    """Sequence b becomes delta[b] tokens longer or shorter (device int32 [num_seqs]).  A partly filled page that others hold is
    copied, in all `pools` (tensors [num_pages, ...]), before its sequence grows out of it."""
    _int32("delta", delta, (pages.num_seqs,), pages.device)
    array, n, bytes_per_page = _pool_list(pages, pools)
    with _on(pages.device, stream):
        ws = pages.refs.new_empty((pages.workspace_bytes + 3) // 4)
        check(lib().cocktail_pages_resize(C.byref(pages.desc), delta.data_ptr(), array, n, bytes_per_page, ws.data_ptr(),
                                          pages.workspace_bytes, _stream_ptr(stream)))


def cocktail_pages_fork(pages: PageTable, source: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Sequence b becomes what sequence source[b] was (device int32 [num_seqs]); source[b] == b leaves it, a negative one frees it."""
    _int32("source", source, (pages.num_seqs,), pages.device)
    with _on(pages.device, stream):
        check(lib().cocktail_pages_fork(C.byref(pages.desc), source.data_ptr(), _stream_ptr(stream)))


def cocktail_pages_compact(pages: PageTable, pools: Sequence[torch.Tensor] = (), stream: Optional[torch.cuda.Stream] = None) -> None:
    """Moves the pages in use to the front of the pools."""
    array, n, bytes_per_page = _pool_list(pages, pools)
    with _on(pages.device, stream):
        ws = pages.refs.new_empty((pages.workspace_bytes + 3) // 4)
        check(lib().cocktail_pages_compact(C.byref(pages.desc), array, n, bytes_per_page, ws.data_ptr(), pages.workspace_bytes,
                                           _stream_ptr(stream)))


def cocktail_pages_check(pages: PageTable, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Waits for the stream and raises CocktailError (code -6) if the last cocktail_pages_resize could not be done."""
    with _on(pages.device, stream):
        check(lib().cocktail_pages_check(C.byref(pages.desc), _stream_ptr(stream)))


def _rows(name: str, t: torch.Tensor, heads: int, head_dim: int, device: torch.device) -> None:
    if t.dtype not in _DTYPES or t.device != device or t.dim() != 3 or tuple(t.shape[1:]) != (heads, head_dim) or t.stride(2) != 1:
        raise TypeError(f"{name} must be a float16 or bfloat16 tensor [tokens, {heads}, {head_dim}] on {device}, channels contiguous")


def _starts(cache: Fp4Cache, starts: Optional[torch.Tensor]) -> Optional[int]:
    if starts is None:
        return None
    _int32("starts", starts, (cache.pages.num_seqs + 1,), cache.pages.device)
    return starts.data_ptr()


def _strides(t: torch.Tensor) -> Tuple[int, int]:
    """Strides of tokens and heads; those of a dimension of one entry say nothing."""
    return (int(t.stride(0)) if t.shape[0] > 1 else t.shape[1] * t.shape[2], int(t.stride(1)) if t.shape[1] > 1 else t.shape[2])


def cocktail_fp4_store(cache: Fp4Cache, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    """Quantizes new tokens into the cache: rows starts[b] .. starts[b+1] of k and v ([tokens, Hkv, D]) become the last tokens of sequence
    b.  Without `starts` every sequence has the same number of rows.  Call cocktail_pages_resize first: it makes the room."""
    dev = cache.pages.device
    _rows("k", k, cache.num_kv_heads, cache.head_dim, dev)
    _rows("v", v, cache.num_kv_heads, cache.head_dim, dev)
    if k.dtype != v.dtype or k.shape != v.shape or _strides(k) != _strides(v):
        raise ValueError("k and v must have the same type, shape and strides")
    st, sh = _strides(k)
    with _on(dev, stream):
        check(lib().cocktail_fp4_store(C.byref(cache.desc), k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype], st, sh, k.shape[0],
                                       _starts(cache, starts), _stream_ptr(stream)))


def cocktail_fp4_gather(cache: Fp4Cache, total: int, starts: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float16,
                        out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream: Optional[torch.cuda.Stream] = None):
    """Reads tokens back as the values they stand for: k, v [total, Hkv, D], rows as in cocktail_fp4_store."""
    dev = cache.pages.device
    with _on(dev, stream):
        if out is None:
            shape = (int(total), cache.num_kv_heads, cache.head_dim)
            out = (torch.empty(shape, dtype=dtype, device=dev), torch.empty(shape, dtype=dtype, device=dev))
        k, v = out
        _rows("k", k, cache.num_kv_heads, cache.head_dim, dev)
        _rows("v", v, cache.num_kv_heads, cache.head_dim, dev)
        if k.dtype != v.dtype or k.shape != v.shape or _strides(k) != _strides(v) or k.shape[0] != total:
            raise ValueError("k and v must have the same type, shape and strides, and `total` rows")
        st, sh = _strides(k)
        check(lib().cocktail_fp4_gather(C.byref(cache.desc), k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype], st, sh, int(total),
                                        _starts(cache, starts), _stream_ptr(stream)))
    return k, v


def cocktail_fp4_attention(cache: Fp4Cache, q: torch.Tensor, starts: Optional[torch.Tensor] = None, max_new: Optional[int] = None,
                           max_len: int = 0, sm_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Causal attention of the newest tokens of every sequence, q [tokens, Hq, D], over the cached keys, themselves included.  Returns
    (out, lse).  max_new: no sequence has more queries (default: as many as there are rows); max_len: about the longest
    sequence, for the split of the work (default: what the table can hold)."""
    dev = cache.pages.device
    if q.dim() != 3:
        raise TypeError("q must be [tokens, Hq, D]")
    total, heads = int(q.shape[0]), int(q.shape[1])
    _rows("q", q, heads, cache.head_dim, dev)
    if max_new is None:
        max_new = total // cache.pages.num_seqs if starts is None else total
    need = C.c_size_t(0)
    st, sh = _strides(q)
    with _on(dev, stream):
        if out is None:
            out = torch.empty((total, heads, cache.head_dim), dtype=q.dtype, device=dev)
        elif out.dtype != q.dtype or out.shape != q.shape or out.device != dev or not out.is_contiguous():
            raise ValueError("out must be a contiguous tensor of q's type, shape and device")
        if lse is None:
            lse = torch.empty((total, heads), dtype=torch.float32, device=dev)
        elif lse.dtype != torch.float32 or tuple(lse.shape) != (total, heads) or lse.device != dev or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32 tensor [tokens, Hq]")
        check(lib().cocktail_fp4_attention_workspace(C.byref(cache.desc), heads, total, int(max_new), int(max_len),
                                                     1 if starts is None else 0, C.byref(need)))
        ws = torch.empty(int(need.value), dtype=torch.uint8, device=dev)
        check(lib().cocktail_fp4_attention(C.byref(cache.desc), heads, q.data_ptr(), _DTYPES[q.dtype], st, sh, total,
                                           _starts(cache, starts), int(max_new), int(max_len), float(sm_scale), out.data_ptr(),
                                           lse.data_ptr(), ws.data_ptr(), int(need.value), _stream_ptr(stream)))
    return out, lse
