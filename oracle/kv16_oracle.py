"""Oracle of the paged 16-bit cache's rotation and of beam search's selection, in binary64 and wider (numpy)."""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import numpy as np


def rotate(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray, interleaved: bool, factor: float = 1.0) -> np.ndarray:
    """x [tokens, heads, D] turned by positions [tokens]: the pairs of the first 2 * len(inv_freq) channels.  Angles in 64 bits of mantissa, reduced by
    whole turns there."""
    n = len(inv_freq)
    turn = 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))
    angle = np.asarray(positions, np.longdouble)[:, None] * np.asarray(inv_freq, np.longdouble)
    angle = (angle - np.rint(angle / turn) * turn)[:, None, :]
    c, s = factor * np.cos(angle).astype(np.float64), factor * np.sin(angle).astype(np.float64)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    out = np.array(x, np.float64)
    u, v = out[..., a].copy(), out[..., b].copy()
    out[..., a], out[..., b] = u * c - v * s, v * c + u * s
    return out


def log_probabilities(row: np.ndarray) -> np.ndarray:
    """Of one row of logits; an infinite logit counts as the largest finite binary32 number, no number as no probability."""
    x = np.array(row, np.float64)
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, float(np.finfo(np.float32).max)))
    top = x.max()
    if top == -np.inf:
        return np.full(len(x), -np.inf)
    return (x - top) - np.log(np.exp(x - top).sum())


def select(logits: np.ndarray, scores: Sequence[float], beams: int, keep: int, eos: int = -1,
           finished: Optional[Sequence[bool]] = None) -> Tuple[np.ndarray, np.ndarray, np.ndarray, np.ndarray]:
    """source, token, score, finished [groups, keep] as include/cocktail.h defines them, candidate by candidate.  (Those of a row are in the order of their
    logits, also where binary64 cannot tell their values apart.)"""
    rows = len(logits)
    result = []
    for first in range(0, rows, beams):
        found: List[Tuple[float, int, float, int, bool]] = []
        for r in range(first, first + beams):
            if not scores[r] > -np.inf:
                continue
            if finished is not None and finished[r]:
                found.append((-float(scores[r]), r, 0.0, eos, True))
                continue
            logp = log_probabilities(logits[r])
            x = np.where(logp > -np.inf, np.minimum(logits[r], float(np.finfo(np.float32).max)), -np.inf)
            best = np.lexsort((np.arange(len(x)), -x))[:keep]              # (no row has more than `keep` of them)
            found += [(-(float(scores[r]) + logp[v]), r, -x[v], int(v), int(v) == eos) for v in best if logp[v] > -np.inf]
        found = sorted(found)[:keep]
        found += [(np.inf, -1, 0.0, -1, False)] * (keep - len(found))
        result.append(found)
    pick = lambda i, dtype: np.array([[c[i] for c in g] for g in result], dtype)  # noqa: E731
    return pick(1, np.int32), pick(3, np.int32), -pick(0, np.float64), pick(4, bool)


def reorder(state: np.ndarray, source: Sequence[int]) -> np.ndarray:
    return np.stack([state[s] if 0 <= s < len(state) else state[r] for r, s in enumerate(source)])
