"""Attention over 16-bit pages where every unit of keys has to be seen in the result: nearly level logits, values that say which unit they belong to, and
bounds that a unit left out or counted twice exceeds (which is tested too, without a GPU)."""
import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck
from oracle import fp4_oracle as F
from test_kv16 import DTYPES, Batch, _f64

gpu = pytest.mark.gpu
UNIT = 32


def marked(t, d, shift=0):
    """Values [t, d]: a one in the channel of the token's unit, zeros elsewhere; `shift` units later."""
    v = np.zeros((t, d))
    v[np.arange(t), (np.arange(t) // UNIT + shift) % d] = 1.0
    return v


def bounds(want, lse, mean_v, size, t, d, dtype, tiles):
    """What a result and its log-sum-exp may be off by.  The result's own rounding; weights that are rounded to the type, in the sum over V and in the normaliser
    (half a step each); logits in binary32, d products and as many sums of terms whose magnitudes sum to `size`, and what it takes to make a weight
    of them (exponent and logarithm, 2^-20, and roundings of the reference); sums in binary32 that one accumulator makes: a step of 32 keys is a term
    of it (with sixteen additions before), at least four waves share a context where there are up to 64 rows, and as many as 512 states are joined.  Weights of fp16
    that are subnormals, by 2^-36 of the largest (2^-32 where there are more than 64 rows), and a result that is one."""
    eps = torch.finfo(dtype).eps / 2
    adds = t // UNIT // (1 if tiles else 4) + 16 + 512
    logit = (d + 4) * 2.0 ** -24 * size + 2.0 ** -21 * (1 + np.abs(lse)) + 2.0 ** -20
    half = dtype == torch.float16
    small = t * 2.0 ** (-32 if tiles else -36) if half else 0.0      # (values are one at most)
    weight = 2 * (eps + logit + adds * 2.0 ** -24)
    return eps * np.abs(want) + weight[..., None] * mean_v * (1 + eps) + small + (2.0 ** -25 if half else 2.0 ** -134), logit + adds * 2.0 ** -24


# ---- the bounds themselves ---------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("t,d,rep", [(33, 64, 1), (1000, 128, 2), (9001, 128, 2), (12345, 128, 8), (20011, 64, 3), (30016, 64, 4), (65536, 128, 1)])
def test_a_unit_that_is_lost_or_counted_twice_is_seen(t, d, rep, dtype):
    """In exact arithmetic, rounded once: the result and the log-sum-exp each exceed their bounds for every unit."""
    rng = np.random.default_rng(t)
    dt = DTYPES[dtype]
    rounded = lambda x: torch.from_numpy(np.array(x)).to(dt).double().numpy()  # noqa: E731
    q, k, v = rounded(rng.standard_normal((1, rep, d)) * 0.5), rounded(rng.standard_normal((t, 1, d))), marked(t, d)[:, None]
    want, lse, mean_v, size = F.attention(q, k, v)
    out_bound, lse_bound = (x[0] for x in bounds(want, lse, mean_v, size, t, d, dt, tiles=True))
    assert (np.abs(rounded(want[0]) - want[0]) <= out_bound).all()
    p = np.exp(q[0] @ k[:, 0].T / np.sqrt(d) - lse[0][:, None])                    # [rep, t]
    for unit in range(-(-t // UNIT)):
        part = p[:, unit * UNIT:(unit + 1) * UNIT].sum(1)
        for times in (-1, 1):
            total = 1 + times * part
            got = want[0].copy()
            got[:, unit % d] += times * part
            with np.errstate(divide="ignore", invalid="ignore"):
                got = rounded(got / total[:, None])
                off = np.abs(np.log(total))
            assert not (np.abs(got - want[0]) <= out_bound).all(1).any(), (unit, times)
            assert (off > lse_bound).all(), (unit, times)


# ---- on the GPU ----------------------------------------------------------------------------------------------------------------------


def check(lens, new, kv_heads, rep, d, page, dtype, max_lens):
    B = Batch(lens, kv_heads, d, page, dtype, seed=len(lens) + sum(lens) % 97)
    for b, t in enumerate(lens):
        for h in range(kv_heads):
            B.v[B.rows(b), h] = torch.from_numpy(marked(t, d, 5 * h + b)).to(B.dev, dtype)
    B.store_all()
    q = B.query(new, rep, 0.5)
    kd, vd, qd = _f64(B.k), _f64(B.v), _f64(q)
    exact, at = [], 0
    for b, n in enumerate(new):
        if n:
            pad = max(0, n - lens[b])
            exact.append((b, at + pad, at + n, F.attention(qd[at + pad:at + n], kd[B.rows(b)], vd[B.rows(b)])))
        at += n
    for max_len in max_lens:
        out, lse = ck.cocktail_kv16_attention(B.cache, q, B.starts(new), max(new), max_len)
        od, ld = _f64(out), _f64(lse)
        for b, lo, hi, (want, wl, mean_v, size) in exact:
            if lens[b] == 0 or lo >= hi:
                continue
            out_bound, lse_bound = bounds(want, wl, mean_v, size, lens[b], d, dtype, max(new) * rep > 64)
            far, off = np.abs(od[lo:hi] - want), np.abs(ld[lo:hi] - wl)
            assert (far <= out_bound).all(), f"sequence {b}, max_len {max_len}: {(far / out_bound).max()} of the bound at {np.argwhere(far > out_bound)[:4].tolist()}"
            assert (off <= lse_bound).all(), f"sequence {b}, max_len {max_len}: lse {(off / lse_bound).max()} of the bound"


CASES = [
    # states of waves and of workgroups, joined by another launch
    ([9001], [1], 1, 2, 128, 16),
    ([33, 20011, 700], [1, 1, 1], 1, 3, 64, 16),
    ([12345, 9000], [1, 1], 1, 8, 128, 48),
    ([4096, 4192, 4096], [1, 1, 1], 1, 1, 128, 64),
    ([5000, 0, 4097], [9, 3, 7], 2, 4, 128, 16),
    ([2048], [16], 1, 4, 64, 16),
    ([3000, 777], [5, 6], 1, 5, 128, 32),
    ([6000 if b in (3, 40, 99) else 10 for b in range(100)], [1 if b in (3, 40, 99) else 0 for b in range(100)], 1, 4, 128, 16),
    ([30000, 40, 30016], [1, 1, 1], 4, 4, 64, 16),
    ([65536], [1], 2, 2, 128, 64),
    # shares of workgroups, segments of workgroups
    ([8000 + 33 * i for i in range(20)], [8] * 20, 2, 6, 128, 16),
    ([300 + 41 * i for i in range(40)], [6] * 40, 2, 8, 64, 16),
    ([31 * i for i in range(60)], [1] * 60, 3, 4, 128, 32),
    ([500, 511, 1, 32, 33], [3] * 5, 4, 16, 128, 16),
    # tiles, whole and with their keys in parts; both kernels in a call
    ([9000], [40], 1, 4, 128, 16),
    ([20011, 700], [70, 33], 1, 2, 64, 48),
    ([3000, 2999], [300, 2999], 2, 1, 128, 16),
    ([8000, 5000, 64], [1, 129, 64], 2, 4, 128, 32),
]


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_every_unit_is_seen_once(case, dtype):
    lens = CASES[case][0]
    check(*CASES[case], DTYPES[dtype], (max(lens), 0, max(lens) // 3, 1))
