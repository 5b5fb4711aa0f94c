"""Binding of the paged 4-bit cache: the page table (cocktail_pages_*) and the cache on top of it (cocktail_fp4_*).

Same names as the C entry points.  torch supplies device memory and streams.  Workspaces: a page table keeps one per stream for the calls that are
made on it and on its caches, one after the other (one for all layers: 17 MB for a step of 8 query rows, 69 MB for 32); what is captured into a graph has one of its own, from the graph's memory, so that graphs and eager calls never
share one.  Threads may call at the same time: a call with a workspace is launched as a whole before the next one begins.  `stream`: another stream
than the current one; it has to be behind what makes the arguments, which may be dropped as soon as the call returns.
"""
from __future__ import annotations

import ctypes as C
import threading
from typing import Optional, Sequence, Tuple

import torch

from . import _lib
from ._lib import check, lib

_DTYPES = {torch.float16: _lib.FP16, torch.bfloat16: _lib.BF16}


def _here(device: torch.device, stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    """Handle of the current stream, if the call is for it and the tensors' device is current; None if that has to be made so (_on)."""
    index = device.index
    return torch._C._cuda_getCurrentRawStream(index) if stream is None and torch._C._cuda_getDevice() == index else None


def _on(device: torch.device, stream: Optional[torch.cuda.Stream]):
    """Makes the tensors' device current for the call, and the stream for what is allocated in it."""
    if stream is None:
        return torch.cuda.device(device)
    if stream.device != device:
        raise ValueError("the stream belongs to another device than the tensors")
    return torch.cuda.stream(stream)


def _used_on(stream: Optional[torch.cuda.Stream], pages: "PageTable", *tensors: Optional[torch.Tensor]) -> None:
    """Behind a call on a stream that it was given: what it works on there may be dropped by the caller at once, and must not be handed out to others
    on its own stream before the call has taken place."""
    if stream is not None:
        for t in (pages.table, pages.seq_lens, pages.refs, pages.status, *tensors):
            if t is not None:
                t.record_stream(stream)


class _Workspaces:
    """Workspaces by stream.  `lock` is held, and the workspace kept, from get() until the call that uses it has returned: a call is several
    launches, and the interpreter lets other threads in between (launches of two calls mixed on one stream would work in the same memory)."""

    def __init__(self, device: torch.device):
        self.device = device
        self.kept = {}
        self.lock = threading.RLock()

    def get(self, need: int, stream: int) -> torch.Tensor:
        """A workspace for a call that is about to be made on the current stream, whose handle is `stream`."""
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(need, dtype=torch.uint8, device=self.device)
        ws = self.kept.get(stream)
        if ws is None or ws.numel() < need:
            ws = self.kept[stream] = torch.empty(need, dtype=torch.uint8, device=self.device)
        return ws


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
        self.num_seqs, self.num_pages = int(table.shape[0]), int(refs.shape[0])
        self.desc = _lib.PageTableDesc(table.data_ptr(), seq_lens.data_ptr(), refs.data_ptr(), status.data_ptr(), table.shape[0],
                                       table.shape[1], page_size, refs.shape[0])
        need = C.c_size_t(0)
        check(lib().cocktail_pages_workspace(C.byref(self.desc), C.byref(need)))   # also checks the sizes
        self.workspace_bytes = int(need.value)
        self.workspaces = _Workspaces(dev)


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
        self.desc_ref = C.byref(self.desc)
        self.workspace_bytes = {}   # by the sizes of the call


_POOL_ARRAYS = {}   # ctypes array types by length


def _pool_list(pages: PageTable, pools: Sequence[torch.Tensor]):
    """ctypes array of the pools' addresses, their number and the bytes of a page."""
    if not pools:
        return None, 0, 0
    index, num_pages, size = pages.device.index, pages.num_pages, pools[0].nbytes
    addresses = []
    for t in pools:
        if t.get_device() != index or not t.is_contiguous() or t.dim() < 1 or t.size(0) != num_pages:
            raise TypeError(f"pools must be contiguous tensors [{num_pages}, ...] on {pages.device}")
        if t.nbytes != size:
            raise ValueError("the pools of a call must have pages of the same size")
        addresses.append(t.data_ptr())
    n = len(addresses)
    array = _POOL_ARRAYS.get(n)
    if array is None:
        array = _POOL_ARRAYS[n] = C.c_void_p * n
    return array(*addresses), n, size // num_pages


def cocktail_pages_resize(pages: PageTable, delta: torch.Tensor, pools: Sequence[torch.Tensor] = (),
                          stream: Optional[torch.cuda.Stream] = None) -> None:
    """Sequence b becomes delta[b] tokens longer or shorter (device int32 [num_seqs]).  A partly filled page that others hold is
    copied, in all `pools` (tensors [num_pages, ...]), before its sequence grows out of it."""
    handle = _here(pages.device, stream)
    if handle is None:
        with _on(pages.device, stream):
            cocktail_pages_resize(pages, delta, pools)
        return _used_on(stream, pages, delta, *pools)
    _int32("delta", delta, (pages.num_seqs,), pages.device)
    array, n, bytes_per_page = _pool_list(pages, pools)
    with pages.workspaces.lock:
        workspace = pages.workspaces.get(pages.workspace_bytes, handle)
        check(lib().cocktail_pages_resize(C.byref(pages.desc), delta.data_ptr(), array, n, bytes_per_page, workspace.data_ptr(),
                                          pages.workspace_bytes, handle))


def cocktail_pages_fork(pages: PageTable, source: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Sequence b becomes what sequence source[b] was (device int32 [num_seqs]); source[b] == b leaves it, a negative one frees it."""
    handle = _here(pages.device, stream)
    if handle is None:
        with _on(pages.device, stream):
            cocktail_pages_fork(pages, source)
        return _used_on(stream, pages, source)
    _int32("source", source, (pages.num_seqs,), pages.device)
    check(lib().cocktail_pages_fork(C.byref(pages.desc), source.data_ptr(), handle))


def cocktail_pages_compact(pages: PageTable, pools: Sequence[torch.Tensor] = (), stream: Optional[torch.cuda.Stream] = None) -> None:
    """Moves the pages in use to the front of the pools."""
    handle = _here(pages.device, stream)
    if handle is None:
        with _on(pages.device, stream):
            cocktail_pages_compact(pages, pools)
        return _used_on(stream, pages, *pools)
    array, n, bytes_per_page = _pool_list(pages, pools)
    with pages.workspaces.lock:
        workspace = pages.workspaces.get(pages.workspace_bytes, handle)
        check(lib().cocktail_pages_compact(C.byref(pages.desc), array, n, bytes_per_page, workspace.data_ptr(), pages.workspace_bytes, handle))


def cocktail_pages_check(pages: PageTable, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Waits for the stream and raises CocktailError (code -6) if the last cocktail_pages_resize could not be done."""
    handle = _here(pages.device, stream)
    if handle is None:
        with _on(pages.device, stream):
            return cocktail_pages_check(pages)
    check(lib().cocktail_pages_check(C.byref(pages.desc), handle))


def _rows(name: str, t: torch.Tensor, heads: int, head_dim: int, device: torch.device) -> Tuple[int, int, int]:
    """Checks rows [tokens, heads, head_dim] and gives their number and their strides of tokens and heads (those of a dimension of one entry
    say nothing)."""
    shape = t.shape
    if t.dtype not in _DTYPES or t.device != device or len(shape) != 3 or shape[1] != heads or shape[2] != head_dim:
        raise TypeError(f"{name} must be a float16 or bfloat16 tensor [tokens, {heads}, {head_dim}] on {device}")
    st, sh, sd = t.stride()
    if sd != 1:
        raise TypeError(f"the channels of {name} must be contiguous")
    return shape[0], st if shape[0] > 1 else heads * head_dim, sh if heads > 1 else head_dim


def _starts(cache: Fp4Cache, starts: Optional[torch.Tensor]) -> Optional[int]:
    if starts is None:
        return None
    if starts.dtype != torch.int32 or starts.device != cache.pages.device or starts.dim() != 1 or \
            starts.shape[0] != cache.pages.num_seqs + 1 or not starts.is_contiguous():
        raise TypeError(f"starts must be a contiguous int32 tensor [{cache.pages.num_seqs + 1}] on {cache.pages.device}")
    return starts.data_ptr()


def cocktail_fp4_store(cache: Fp4Cache, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    """Quantizes new tokens into the cache: rows starts[b] .. starts[b+1] of k and v ([tokens, Hkv, D]) become the last tokens of sequence
    b.  Without `starts` every sequence has the same number of rows.  Call cocktail_pages_resize first: it makes the room."""
    dev = cache.pages.device
    handle = _here(dev, stream)
    if handle is None:
        with _on(dev, stream):
            cocktail_fp4_store(cache, k, v, starts)
        return _used_on(stream, cache.pages, cache.pool, k, v, starts)
    rows = _rows("k", k, cache.num_kv_heads, cache.head_dim, dev)
    if rows != _rows("v", v, cache.num_kv_heads, cache.head_dim, dev) or k.dtype != v.dtype:
        raise ValueError("k and v must have the same type, shape and strides")
    check(lib().cocktail_fp4_store(cache.desc_ref, k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype], rows[1], rows[2], rows[0],
                                   _starts(cache, starts), handle))


def cocktail_fp4_gather(cache: Fp4Cache, total: int, starts: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float16,
                        out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream: Optional[torch.cuda.Stream] = None):
    """Reads tokens back as the values they stand for: k, v [total, Hkv, D], rows as in cocktail_fp4_store."""
    dev = cache.pages.device
    handle = _here(dev, stream)
    if handle is None:
        with _on(dev, stream):
            result = cocktail_fp4_gather(cache, total, starts, dtype, out)
        _used_on(stream, cache.pages, cache.pool, starts, *(out or ()))
        return result
    if out is None:
        shape = (int(total), cache.num_kv_heads, cache.head_dim)
        out = (torch.empty(shape, dtype=dtype, device=dev), torch.empty(shape, dtype=dtype, device=dev))
    k, v = out
    rows = _rows("k", k, cache.num_kv_heads, cache.head_dim, dev)
    if rows != _rows("v", v, cache.num_kv_heads, cache.head_dim, dev) or k.dtype != v.dtype or rows[0] != total:
        raise ValueError("k and v must have the same type, shape and strides, and `total` rows")
    check(lib().cocktail_fp4_gather(cache.desc_ref, k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype], rows[1], rows[2], rows[0],
                                    _starts(cache, starts), handle))
    return k, v


def cocktail_fp4_attention(cache: Fp4Cache, q: torch.Tensor, starts: Optional[torch.Tensor] = None, max_new: Optional[int] = None,
                           max_len: int = 0, sm_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Causal attention of the newest tokens of every sequence, q [tokens, Hq, D], over the cached keys, themselves included.  Returns
    (out, lse).  max_new: no sequence has more queries (default: as many as there are rows); max_len: about the longest
    sequence, for the split of the work (default: what the table can hold)."""
    dev = cache.pages.device
    handle = _here(dev, stream)
    if handle is None:
        with _on(dev, stream):
            result = cocktail_fp4_attention(cache, q, starts, max_new, max_len, sm_scale, out, lse)
        _used_on(stream, cache.pages, cache.pool, q, starts, out, lse)
        return result
    if q.dim() != 3:
        raise TypeError("q must be [tokens, Hq, D]")
    heads = q.shape[1]
    total, st, sh = _rows("q", q, heads, cache.head_dim, dev)
    if max_new is None:
        max_new = total // cache.pages.num_seqs if starts is None else total
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.dtype != q.dtype or out.shape != q.shape or out.device != dev or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of q's type, shape and device")
    if lse is None:
        lse = q.new_empty((total, heads), dtype=torch.float32)
    elif lse.dtype != torch.float32 or tuple(lse.shape) != (total, heads) or lse.device != dev or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 tensor [tokens, Hq]")
    first = _starts(cache, starts)
    key = (heads, total, max_new, max_len, starts is None)
    need = cache.workspace_bytes.get(key)
    if need is None:
        size = C.c_size_t(0)
        check(lib().cocktail_fp4_attention_workspace(cache.desc_ref, heads, total, int(max_new), int(max_len),
                                                     1 if starts is None else 0, C.byref(size)))
        if len(cache.workspace_bytes) > 4096:
            cache.workspace_bytes.clear()
        need = cache.workspace_bytes[key] = int(size.value)
    workspaces = cache.pages.workspaces
    with workspaces.lock:
        workspace = workspaces.get(need, handle)
        check(lib().cocktail_fp4_attention(cache.desc_ref, heads, q.data_ptr(), _DTYPES[q.dtype], st, sh, total, first, int(max_new), int(max_len),
                                           float(sm_scale), out.data_ptr(), lse.data_ptr(), workspace.data_ptr(), need, handle))
    return out, lse
