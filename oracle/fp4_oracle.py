"""CPU oracle of the paged 4-bit cache: quantizer, page layout, attention in binary64, page bookkeeping by walking through the rows.

Test infrastructure only; written from include/cocktail.h, shares no code with the library.
"""
from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def quantize(x: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """x: [..., D] in any float type.  (codes uint8 [..., D] in 0..15, scale bytes uint8 [..., D/32])."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, GROUP)
    g = np.where(np.isnan(g), 0.0, g)
    top = np.minimum(np.abs(g).max(axis=-1, keepdims=True), 1e300)
    # frexp: top = f * 2^x with 0.5 <= f < 1
    e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1 - 2, -23)
    e = np.clip(e, -23, 13)
    a = np.minimum(np.minimum(np.abs(g), 1e300) / 2.0 ** e, 100.0)
    # nearest magnitude, ties to the even number
    dist = np.abs(a[..., None] - MAGNITUDES)
    best = dist.min(axis=-1, keepdims=True)
    near = dist == best
    low = near.argmax(axis=-1)
    both = near.sum(axis=-1) == 2
    number = np.where(both & (low % 2 == 1), low + 1, low)
    code = (number + 8 * np.signbit(g)).astype(np.uint8)
    return code.reshape(x.shape), (e[..., 0] + 127).astype(np.uint8)


def dequantize(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    v = np.where(codes >= 8, -1.0, 1.0) * MAGNITUDES[codes & 7]
    g = v.reshape(*codes.shape[:-1], -1, GROUP) * 2.0 ** (scales.astype(np.float64) - 127)[..., None]
    return g.reshape(codes.shape)


def value(x: np.ndarray) -> np.ndarray:
    return dequantize(*quantize(x))


def run_bytes(head_dim: int, page_size: int) -> int:
    return page_size * (head_dim + head_dim // 16)


def put(pool: np.ndarray, page: int, at: int, head: int, head_dim: int, page_size: int, k: np.ndarray, v: np.ndarray) -> None:
    """Writes one token's row of one head (k, v: [D]) into pool [pages, bytes], byte by byte as the layout says."""
    base = head * run_bytes(head_dim, page_size)
    kc, ks = quantize(k)
    vc, vs = quantize(v)
    p = pool[page]
    for y in range(head_dim // 2):
        p[base + at * head_dim // 2 + y] = kc[2 * y] | kc[2 * y + 1] << 4
        p[base + page_size * head_dim // 2 + (at // 4) * 2 * head_dim + (y // 4) * 16 + (at % 4) * 4 + y % 4] = vc[2 * y] | vc[2 * y + 1] << 4
    for g in range(head_dim // GROUP):
        p[base + page_size * head_dim + at * (head_dim // GROUP) + g] = ks[g]
        p[base + page_size * head_dim + page_size * head_dim // GROUP + (at // 4) * (head_dim // 8) + g * 4 + at % 4] = vs[g]


def get(pool: np.ndarray, page: int, at: int, head: int, head_dim: int, page_size: int) -> Tuple[np.ndarray, np.ndarray]:
    """The values of one token's row of one head."""
    base = head * run_bytes(head_dim, page_size)
    p = pool[page]
    y = np.arange(head_dim // 2)
    kb = p[base + at * head_dim // 2 + y]
    vb = p[base + page_size * head_dim // 2 + (at // 4) * 2 * head_dim + (y // 4) * 16 + (at % 4) * 4 + y % 4]
    g = np.arange(head_dim // GROUP)
    ks = p[base + page_size * head_dim + at * (head_dim // GROUP) + g]
    vs = p[base + page_size * head_dim + page_size * head_dim // GROUP + (at // 4) * (head_dim // 8) + g * 4 + at % 4]
    split = lambda b: np.stack([b & 15, b >> 4], axis=-1).reshape(-1)  # noqa: E731
    return dequantize(split(kb), ks), dequantize(split(vb), vs)


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, keep: Optional[np.ndarray] = None, sm_scale: Optional[float] = None):
    """q: [n, Hq, D]; k, v: [T, Hkv, D] (values), the last n of them the queries' own; keep: bool [T], tokens that exist.
    (out [n, Hq, D], lse [n, Hq], and what bounds a computed result: weights' mean |v| [n, Hq, D], largest sum |q||k| [n, Hq])."""
    n, hq, d = q.shape
    t, hkv = k.shape[0], k.shape[1]
    scale = 1 / math.sqrt(d) if not sm_scale or sm_scale <= 0 else sm_scale
    kk, vv = (np.repeat(x.astype(np.float64), hq // hkv, axis=1).transpose(1, 0, 2) for x in (k, v))        # [Hq, T, D]
    qq = q.astype(np.float64).transpose(1, 0, 2)                                                            # [Hq, n, D]
    seen = np.arange(t)[None, :] <= (t - n + np.arange(n))[:, None]
    if keep is not None:
        seen = seen & keep[None, :]
    s = np.where(seen[None], qq @ kk.transpose(0, 2, 1) * scale, -np.inf)
    if t == 0:
        zero = np.zeros((n, hq, d))
        return zero, np.full((n, hq), -np.inf), zero, np.zeros((n, hq))
    top = s.max(axis=-1, keepdims=True)
    w = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    total = w.sum(axis=-1, keepdims=True)
    safe = np.where(total > 0, total, 1.0)
    with np.errstate(divide="ignore"):
        lse = np.where(total > 0, top + np.log(total), -np.inf)[..., 0]
    size = np.where(seen[None], np.abs(qq) @ np.abs(kk).transpose(0, 2, 1) * scale, 0.0).max(axis=-1)
    tr = lambda x: np.moveaxis(x, 0, 1)  # noqa: E731
    return tr(w / safe @ vv), tr(lse), tr(w / safe @ np.abs(vv)), tr(size)


class Pages:
    """The page table as lists; every operation walks through the rows as include/cocktail.h tells it."""

    def __init__(self, num_seqs: int, stride: int, num_pages: int, page_size: int):
        self.rows: List[List[int]] = [[] for _ in range(num_seqs)]
        self.lens = [0] * num_seqs
        self.refs = [0] * num_pages
        self.stride, self.page_size, self.status = stride, page_size, 0

    def table(self) -> np.ndarray:
        return np.array([r + [-1] * (self.stride - len(r)) for r in self.rows], dtype=np.int32)

    def resize(self, delta: Sequence[int], pools: bool = True) -> List[Tuple[int, int]]:
        ps = self.page_size
        free = [i for i, r in enumerate(self.refs) if r == 0]
        rows, refs, lens, moves, taken = [list(r) for r in self.rows], list(self.refs), list(self.lens), [], 0
        for b, d in enumerate(delta):
            if lens[b] + max(0, d) > self.stride * ps:
                self.status = -1
                return []
        # pages that a row shares with rows that shrink now are shared all the same
        held = list(self.refs)
        for b, d in enumerate(delta):
            after = max(0, lens[b] + d)
            need = -(-after // ps)
            if d > 0 and lens[b] % ps and held[rows[b][-1]] > 1:
                old = rows[b][-1]
                held[old] -= 1
                refs[old] -= 1
                if taken < len(free):
                    rows[b][-1] = free[taken]
                    refs[free[taken]] = 1
                    moves.append((old, free[taken]))
                taken += 1
            while len(rows[b]) < need:
                if taken < len(free):
                    refs[free[taken]] = 1
                rows[b].append(free[taken] if taken < len(free) else -7)
                taken += 1
            for page in rows[b][need:]:
                refs[page] -= 1
            del rows[b][need:]
            lens[b] = after
        if moves and not pools:
            self.status = -2
            return []
        if taken > len(free):
            self.status = taken - len(free)
            return []
        self.rows, self.refs, self.lens, self.status = rows, refs, lens, 0
        return moves

    def _recount(self) -> None:
        self.refs = [0] * len(self.refs)
        for r in self.rows:
            for page in r:
                self.refs[page] += 1

    def fork(self, source: Sequence[int]) -> None:
        old, lens, n = [list(r) for r in self.rows], list(self.lens), len(self.rows)
        for b, s in enumerate(source):
            if s < n and s != b:
                self.rows[b], self.lens[b] = (list(old[s]), lens[s]) if s >= 0 else ([], 0)
        self._recount()

    def compact(self) -> List[Tuple[int, int]]:
        n = sum(r > 0 for r in self.refs)
        moves = list(zip([i for i in range(n, len(self.refs)) if self.refs[i]], [i for i in range(n) if not self.refs[i]]))
        to = dict(moves)
        self.rows = [[to.get(i, i) for i in r] for r in self.rows]
        self._recount()
        return moves
