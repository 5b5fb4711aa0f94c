"""Binding of a step of beam search (cocktail_beam_*): selection over hypotheses and vocabulary, and the reordering of what hypotheses carry (their pages
follow with cocktail_pages_fork).

Same names as the C entry points.  A call's workspace is allocated for it, so that calls on different streams, threads and in graphs share none.
`stream`: another stream than the current one; it has to be behind what makes the arguments, which may be dropped as soon as the call returns.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple

import torch

from . import _lib
from ._lib import check, lib
from .paged import _here, _on

_LOGITS = {torch.float16: _lib.FP16, torch.bfloat16: _lib.BF16, torch.float32: _lib.FP32}
_NEEDS = {}   # bytes of the workspace by sizes


def _record(stream: Optional[torch.cuda.Stream], *tensors: Optional[torch.Tensor]) -> None:
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def _vector(name: str, t: torch.Tensor, dtypes, n: int, device: torch.device) -> None:
    if t.dtype not in dtypes or t.device != device or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {' or '.join(str(d)[6:] for d in dtypes)} tensor of {n} on {device}")


def cocktail_beam_select(logits: torch.Tensor, scores: torch.Tensor, beams: int, keep: Optional[int] = None, eos: int = -1,
                         finished: Optional[torch.Tensor] = None,
                         out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                         stream: Optional[torch.cuda.Stream] = None):
    """Selects the `keep` (default: `beams`) best continuations of every request.  logits [requests * beams, vocab] (float16, bfloat16 or float32, rows
    may be strided), scores float32 [requests * beams]: log probabilities of the hypotheses; finished (bool or uint8 [requests * beams]): those that
    have ended, and have `eos` at their own score as their only continuation.
    Returns (source, token, score, finished), [requests, keep] each, best first: rows of logits (int32), tokens (int32), log probabilities (float32), and
    which continuations have ended (bool); -1, -1, -inf and False where a request has no further ones.  out: these four, to be written into."""
    if not logits.is_cuda or logits.dim() != 2 or logits.dtype not in _LOGITS or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise TypeError("logits must be a float16, bfloat16 or float32 device tensor [requests * beams, vocab] with contiguous rows")
    dev = logits.device
    handle = _here(dev, stream)
    if handle is None:
        with _on(dev, stream):
            result = cocktail_beam_select(logits, scores, beams, keep, eos, finished, out)
        _record(stream, logits, scores, finished, *result)
        return result
    rows, vocab = logits.shape
    beams = int(beams)
    keep = beams if keep is None else int(keep)
    if beams < 1 or rows < 1 or rows % beams:
        raise ValueError("the rows of logits must be a positive multiple of beams")
    groups = rows // beams
    _vector("scores", scores, (torch.float32,), rows, dev)
    if finished is not None:
        _vector("finished", finished, (torch.bool, torch.uint8), rows, dev)
    key = (groups, beams, vocab, keep)
    need = _NEEDS.get(key)
    if need is None:
        size = C.c_size_t(0)
        check(lib().cocktail_beam_select_workspace(groups, beams, vocab, keep, C.byref(size)))
        if len(_NEEDS) > 4096:
            _NEEDS.clear()
        need = _NEEDS[key] = int(size.value)
    if out is None:
        # (empty_strided: the call costs less on the host than the others that make a tensor, 1.3 of 1.7 us, and small steps are as long as the host takes)
        size, strides, make = (groups, keep), (keep, 1), torch.empty_strided
        source, token = make(size, strides, dtype=torch.int32, device=dev), make(size, strides, dtype=torch.int32, device=dev)
        score, ended = make(size, strides, dtype=torch.float32, device=dev), make(size, strides, dtype=torch.bool, device=dev)
    else:
        source, token, score, ended = out
        _vector("source", source, (torch.int32,), groups * keep, dev)
        _vector("token", token, (torch.int32,), groups * keep, dev)
        _vector("score", score, (torch.float32,), groups * keep, dev)
        _vector("finished", ended, (torch.bool, torch.uint8), groups * keep, dev)
    workspace = torch.empty_strided((need,), (1,), dtype=torch.uint8, device=dev)
    check(lib().cocktail_beam_select(logits.data_ptr(), _LOGITS[logits.dtype], logits.stride(0) if rows > 1 else vocab, groups, beams, vocab, keep,
                                     scores.data_ptr(), finished.data_ptr() if finished is not None else None, int(eos), source.data_ptr(),
                                     token.data_ptr(), score.data_ptr(), ended.data_ptr(), workspace.data_ptr(), need, handle))
    return source, token, score, ended


_ARRAYS = {}   # ctypes array types by length


def _overlap(written, read) -> bool:
    """Whether one of the spans (first, end) that are written has bytes in common with another one, or with one that is read."""
    spans = sorted([(a, b, True) for a, b in written if b > a] + [(a, b, False) for a, b in read if b > a])
    end_written = end_read = 0
    for first, end, own in spans:
        if first < end_written or (own and first < end_read):
            return True
        if own:
            end_written = max(end_written, end)
        else:
            end_read = max(end_read, end)
    return False


def cocktail_beam_reorder(source: torch.Tensor, states: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None,
                          stream: Optional[torch.cuda.Stream] = None):
    """Row r of every state (contiguous tensors [rows, ...]) becomes what row source[r] was (device int32 of `rows` entries); rows whose source is negative
    stay as they are.  In place, or into the tensors of `out`, which must not overlap with the states.  Returns the reordered tensors."""
    if not source.is_cuda:
        raise TypeError("source must be a device tensor")
    dev = source.device
    handle = _here(dev, stream)
    if handle is None:
        with _on(dev, stream):
            result = cocktail_beam_reorder(source, states, out)
        _record(stream, source, *states, *result)
        return result
    rows = source.numel()
    _vector("source", source, (torch.int32,), rows, dev)
    if rows < 1:
        raise ValueError("source must have a row at least")
    states = list(states)
    result = states if out is None else list(out)
    n, index = len(states), dev.index
    if len(result) != n:
        raise ValueError("out must have a tensor for every state")
    first = source.data_ptr()
    read, written, sizes = [(first, first + 4 * rows)], [], []
    for t, o in zip(states, result):
        if t.get_device() != index or not t.is_contiguous() or t.dim() < 1 or t.size(0) != rows:
            raise TypeError(f"states must be contiguous tensors [{rows}, ...] on {dev}")
        size, at = t.nbytes, t.data_ptr()
        sizes.append(size // rows)
        if o is not t:
            if o.get_device() != index or not o.is_contiguous():
                raise TypeError(f"out must have contiguous tensors on {dev}")
            if o.dtype != t.dtype or o.shape != t.shape:
                raise ValueError("out must have the states' types and shapes")
            read.append((at, at + size))
            at = o.data_ptr()
        written.append((at, at + size))
    if n and _overlap(written, read):
        raise ValueError("states that are written must not overlap with others or with the sources")
    arrays = _ARRAYS.get(n)
    if arrays is None:
        arrays = _ARRAYS[n] = C.c_void_p * n, C.c_int64 * n
    to = arrays[0](*[a for a, _ in written])
    of = to if len(read) == 1 else arrays[0](*[t.data_ptr() for t in states])   # (all of them in place)
    check(lib().cocktail_beam_reorder(first, rows, of, to, arrays[1](*sizes), n, handle))
    return result
