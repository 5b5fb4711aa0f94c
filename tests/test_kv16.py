"""The paged 16-bit cache: appending with the rotation, and attention, against the oracle in binary64."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck
from oracle import fp4_oracle as F
from oracle import kv16_oracle as O
from paper_2503_23294_amd import _lib

gpu = pytest.mark.gpu
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _f64(t):
    return t.detach().cpu().double().numpy()


# ---- without a GPU: the oracle against facts of its own, and every refusal of the C entry points ---------------------------------


def test_rotation_of_the_oracle():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 2, 64))
    freq = 10000.0 ** (-np.arange(16) / 16)
    for interleaved in (False, True):
        assert np.array_equal(O.rotate(x, np.zeros(5), freq, interleaved), x)                 # position 0: as it is
        y = O.rotate(x, [3, -7, 10 ** 6, 2 ** 31 - 1, 12], freq, interleaved)
        assert np.array_equal(y[..., 32:], x[..., 32:]) and np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        back = O.rotate(y, [-3, 7, -10 ** 6, 1 - 2 ** 31, -12], freq, interleaved)
        assert np.allclose(back, x, atol=1e-12)
        # products depend on the distance alone
        q, k = rng.standard_normal((2, 1, 1, 64))
        dots = [(O.rotate(q, [p], freq, interleaved) * O.rotate(k, [p - 5], freq, interleaved)).sum() for p in (5, 100, 4096)]
        assert np.ptp(dots) < 1e-10
    quarter = O.rotate(np.array([[[1.0, 0.0]]]), [1], [np.pi / 2], True, factor=2.0)
    assert np.allclose(quarter, [[[0.0, 2.0]]], atol=1e-15)


def _desc(**more):
    d = dict(table=4096, seq_lens=4096, refs=4096, status=4096, num_seqs=4, table_stride=8, page_size=16, num_pages=32)
    d.update(more)
    return _lib.PageTableDesc(*d.values())


def _cache_desc(k=4096, v=1 << 20, heads=2, head_dim=128, dtype=0, **more):
    return _lib.Kv16CacheDesc(_desc(**more), k, v, heads, head_dim, dtype, 0)


BAD_CACHES = [(dict(head_dim=80), _lib.EUNSUPPORTED), (dict(k=None), _lib.EINVAL), (dict(v=None), _lib.EINVAL), (dict(k=8), _lib.EALIGN),
              (dict(v=4104), _lib.EALIGN), (dict(page_size=8), _lib.EINVAL), (dict(page_size=24), _lib.EINVAL), (dict(page_size=1 << 17), _lib.EINVAL),
              (dict(heads=0), _lib.EINVAL), (dict(heads=1025), _lib.EINVAL), (dict(dtype=2), _lib.EINVAL), (dict(num_seqs=0), _lib.EINVAL),
              (dict(table_stride=(1 << 27) - 1), _lib.EINVAL), (dict(table=None), _lib.EINVAL)]


def _append(L, c=None, k=4096, v=4096, st=256, sh=128, total=8, starts=4096, rot=(4096, 128, 0, 1.0), pos=None, q=4096, hq=4, qst=512, qsh=128, out=1 << 21):
    r = None if rot is None else C.byref(_lib.RotationDesc(*rot, 0))
    return L.cocktail_kv16_append(C.byref(c or _cache_desc()), k, v, st, sh, total, starts, r, pos, q, hq, qst, qsh, out, None)


def test_refusals_of_append():
    L = _lib.lib()
    for bad, code in BAD_CACHES:
        assert _append(L, c=_cache_desc(**bad)) == code, bad
    assert L.cocktail_kv16_append(None, 4096, 4096, 256, 128, 8, None, None, None, None, 0, 0, 0, None, None) == _lib.EINVAL
    for more, code in ((dict(k=None), _lib.EINVAL), (dict(v=None), _lib.EINVAL), (dict(k=8), _lib.EALIGN), (dict(st=130), _lib.EINVAL), (dict(st=-256), _lib.EINVAL),
                       (dict(sh=4), _lib.EINVAL), (dict(st=120), _lib.EINVAL), (dict(sh=64), _lib.EINVAL), (dict(total=-1), _lib.EINVAL),
                       (dict(total=(1 << 30) + 1), _lib.EINVAL), (dict(total=1 << 29), _lib.EINVAL), (dict(starts=2), _lib.EALIGN),
                       (dict(total=6, starts=None), _lib.EINVAL), (dict(pos=2), _lib.EALIGN),
                       (dict(rot=(None, 128, 0, 1.0)), _lib.EINVAL), (dict(rot=(4100, 128, 0, 1.0)), _lib.EALIGN), (dict(rot=(4096, 0, 0, 1.0)), _lib.EUNSUPPORTED),
                       (dict(rot=(4096, 144, 0, 1.0)), _lib.EUNSUPPORTED), (dict(rot=(4096, 24, 0, 1.0)), _lib.EUNSUPPORTED),
                       (dict(rot=(4096, 64, 2, 1.0)), _lib.EINVAL), (dict(rot=(4096, 64, 1, float("inf"))), _lib.EINVAL),
                       (dict(rot=None), _lib.EINVAL), (dict(rot=None, q=None, hq=0, out=None, pos=4096), _lib.EINVAL),
                       (dict(hq=0), _lib.EINVAL), (dict(hq=65537), _lib.EINVAL), (dict(out=None), _lib.EINVAL), (dict(q=8), _lib.EALIGN), (dict(out=8), _lib.EALIGN),
                       (dict(qst=516), _lib.EINVAL), (dict(qsh=64), _lib.EINVAL), (dict(q=None), _lib.EINVAL), (dict(q=None, hq=0), _lib.EINVAL),
                       (dict(out=4096, qst=1024), _lib.EINVAL), (dict(out=4096, qst=512, qsh=136), _lib.EINVAL)):
        assert _append(L, **more) == code, more
        assert L.cocktail_last_error()
    # nothing to do: nothing is launched
    assert _append(L, total=0) == 0 and _append(L, total=0, rot=None, q=None, hq=0, out=None) == 0


def test_refusals_of_attention():
    L = _lib.lib()
    n = C.c_size_t(0)

    def call(c=None, hq=4, q=4096, st=512, sh=128, total=8, starts=4096, max_new=8, max_len=0, scale=0.0, out=4096, lse=None, ws=4096, wb=1 << 40):
        return L.cocktail_kv16_attention(C.byref(c or _cache_desc()), hq, q, st, sh, total, starts, max_new, max_len, scale, out, lse, ws, wb, None)
    for bad, code in BAD_CACHES:
        assert call(c=_cache_desc(**bad)) == code, bad
        assert L.cocktail_kv16_attention_workspace(C.byref(_cache_desc(**bad)), 4, 8, 8, 0, 0, C.byref(n)) == code, bad
    assert L.cocktail_kv16_attention_workspace(C.byref(_cache_desc()), 4, 8, 8, 0, 0, C.byref(n)) == 0 and n.value > 0
    assert L.cocktail_kv16_attention_workspace(C.byref(_cache_desc()), 4, 8, 8, 0, 0, None) == _lib.EINVAL
    assert call(wb=n.value - 1) == _lib.ENOSPACE
    assert call(hq=3) == _lib.EINVAL and call(hq=0) == _lib.EINVAL and call(hq=130) == _lib.EUNSUPPORTED
    assert call(q=None) == _lib.EINVAL and call(out=None) == _lib.EINVAL and call(q=4104) == _lib.EALIGN
    assert call(max_new=0) == _lib.EINVAL and call(max_new=9) == _lib.EINVAL and call(total=-1) == _lib.EINVAL
    assert call(total=1 << 29, max_new=1) == _lib.EINVAL
    assert call(starts=None, max_new=3) == _lib.EINVAL and call(total=6, starts=None, max_new=1) == _lib.EINVAL
    assert call(scale=float("nan")) == _lib.EINVAL and call(scale=float("inf")) == _lib.EINVAL
    assert call(ws=None) == _lib.EINVAL and call(ws=8) == _lib.EALIGN and call(lse=2) == _lib.EALIGN
    assert call(c=_cache_desc(num_seqs=15, table_stride=(1 << 27) - 16, page_size=16)) == _lib.EINVAL   # more units than are numbered
    assert call(total=0, max_new=0) == 0


# ---- on the GPU ------------------------------------------------------------------------------------------------------------


class Batch:
    """A cache whose pages lie in random places of pools full of junk (infinities and NaN among it), and the tokens that belong into it."""

    def __init__(self, lens, kv_heads, head_dim, page, dtype, seed=0, spread=1.0, spare=3, columns=0):
        self.dev = torch.device("cuda:0")
        self.lens, self.h, self.d, self.page, self.dtype = list(lens), kv_heads, head_dim, page, dtype
        rng = np.random.default_rng(seed)
        need = [-(-t // page) for t in lens]
        pages = sum(need) + spare
        ids = rng.permutation(pages).astype(np.int32)
        # room for long contexts, so that calls that name no length are cut as for those
        table = np.full((len(lens), columns or max(max(need) + 1, 20000 // page)), -1, np.int32)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = ids[at:at + k]
            at += k
        refs = np.zeros(pages, np.int32)
        refs[ids[:at]] = 1
        self.table = table
        t = lambda a: torch.from_numpy(a).to(self.dev)  # noqa: E731
        self.pages = ck.PageTable.of(t(table), t(np.array(lens, np.int32)), t(refs), page)
        self.cache = ck.Kv16Cache(self.pages, kv_heads, head_dim, dtype)
        for pool in self.cache.pools:
            junk = rng.integers(0, 65536, tuple(pool.shape), dtype=np.uint16)
            junk[rng.random(junk.shape) < 0.2] = 0x7fff                                # NaN in either type
            pool.view(torch.int16).copy_(t(junk.view(np.int16)))
        make = lambda: torch.from_numpy(rng.standard_normal((sum(lens), kv_heads, head_dim)) * spread ** rng.uniform(-1, 1, (sum(lens), kv_heads, 1))).to(self.dev, dtype)  # noqa: E731
        self.k, self.v = make(), make()
        self.rng = rng

    def starts(self, counts):
        return torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(self.dev)

    def store_all(self):
        ck.cocktail_kv16_append(self.cache, self.k, self.v, self.starts(self.lens))

    def rows(self, b):
        at = sum(self.lens[:b])
        return slice(at, at + self.lens[b])

    def query(self, new, rep, scale=1.0):
        return torch.from_numpy(self.rng.standard_normal((sum(new), self.h * rep, self.d)) * scale).to(self.dev, self.dtype)

    def pool_rows(self, b, lo, hi, pool):
        """Tokens lo .. hi-1 of sequence b as the pool has them [tokens, heads, D]."""
        pos = np.arange(lo, hi)
        page = torch.from_numpy(self.table[b, pos // self.page].astype(np.int64)).to(self.dev)
        return pool[page, :, torch.from_numpy(pos % self.page).to(self.dev)]

    def check(self, q, new, out, lse, sm_scale=None, keep=None):
        """Against binary64.  Bounds: the result's own rounding (half a step); weights rounded to the type, in the sum over V and in the normaliser (half a
        step each at most), and, where they are fp16 subnormals, by 2^-25 of the reference; logits: D products and sums in binary32 of
        terms whose magnitudes sum to `size`; sums over the keys in binary32."""
        eps = torch.finfo(q.dtype).eps / 2
        qd, kd, vd, od, ld = _f64(q), _f64(self.k), _f64(self.v), _f64(out), _f64(lse)
        at = 0
        for b, n in enumerate(new):
            if not n:
                continue
            t, r = self.lens[b], self.rows(b)
            kb, vb, qb = kd[r], vd[r], qd[at:at + n]
            pad = max(0, n - t)      # queries before the first token
            want, wl, mean_v, size = F.attention(qb[pad:], kb, vb, None if keep is None else keep[b], sm_scale)
            got, gl = od[at:at + n], ld[at:at + n]
            assert (got[:pad] == 0).all() and np.isneginf(gl[:pad]).all(), f"sequence {b}: queries without keys"
            got, gl = got[pad:], gl[pad:]
            none = np.isneginf(wl)
            assert (got[none] == 0).all() and (np.isneginf(gl) == none).all(), f"sequence {b}: rows without keys"
            logit = (self.d + 4) * 2.0 ** -24 * size + 2.0 ** -21 * (1 + np.abs(np.where(none, 0, wl))) + 2.0 ** -20
            weight = 2 * (eps + logit + t * 2.0 ** -24)
            bound = eps * np.abs(want) + weight[..., None] * mean_v * (1 + eps) + t * 2.0 ** -25 * (np.abs(vb).max() if t else 0) + 2.0 ** -25
            far = np.abs(got - want)
            assert (far <= bound).all(), f"sequence {b}: {np.max(far - bound)} over, {np.max(far)} off, at {np.argwhere(far > bound)[:4].tolist()}"
            far = np.abs(np.where(none, 0, gl) - np.where(none, 0, wl))
            assert (far <= logit + t * 2.0 ** -24).all(), f"sequence {b}: lse off by {far.max()}"
            at += n


def _freq(rotary, base=10000.0):
    return base ** (-2.0 * np.arange(rotary // 2) / rotary)


def _rotation(rotary, interleaved=False, factor=1.0, base=10000.0):
    return ck.Rotation(torch.from_numpy(_freq(rotary, base)).cuda(), interleaved, factor)


def _check_turned(got, x, positions, freq, interleaved, factor, dtype):
    """Bounds: sine and cosine within pi * 2^-24 (the angle as binary32) and 2^-22 (the functions), four roundings of binary32 in products and sums, and
    the result's own."""
    want = O.rotate(_f64(x), positions, freq, interleaved, factor)
    n = len(freq)
    a = np.abs(_f64(x))
    size = a.copy()
    u, v = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    size[..., u] = size[..., v] = a[..., u] + a[..., v]
    bound = torch.finfo(dtype).eps / 2 * np.abs(want) + 12 * 2.0 ** -24 * abs(factor) * size + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)
    bound[..., 2 * n:] = 0
    far = np.abs(_f64(got) - want)
    assert (far <= bound).all(), f"{np.max(far - bound)} over at {np.argwhere(far > bound)[:4].tolist()}"


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,rep,d,page,rotary,interleaved,factor", [(2, 4, 128, 16, 128, False, 1.0), (3, 1, 64, 48, 64, True, 1.0), (1, 5, 128, 64, 32, True, 1.25),
                                                                       (5, 2, 64, 16, 16, False, 0.5), (1, 1, 128, 32, 96, False, 1.0), (2, 3, 64, 16, 48, False, -1.0)])
def test_append_rotates_and_writes_nothing_else(heads, rep, d, page, rotary, interleaved, factor, dtype):
    lens, new = [37, 1, 0, 200, 64, 16], [37, 1, 0, 3, 17, 0]
    B = Batch(lens, heads, d, page, DTYPES[dtype], seed=d + page)
    k, v = (torch.from_numpy(B.rng.standard_normal((sum(new), heads, d))).to(B.dev, B.dtype) for _ in range(2))
    q = B.query(new, rep)
    before = [p.clone() for p in B.cache.pools]
    rot = _rotation(rotary, interleaved, factor)
    out = ck.cocktail_kv16_append(B.cache, k, v, B.starts(new), rot, q=q)
    positions = np.concatenate([np.arange(t - n, t) for t, n in zip(lens, new)])
    _check_turned(out, q, positions, _freq(rotary), interleaved, factor, B.dtype)
    got = [torch.cat([B.pool_rows(b, t - n, t, p) for b, (t, n) in enumerate(zip(lens, new))]) for p in B.cache.pools]
    _check_turned(got[0], k, positions, _freq(rotary), interleaved, factor, B.dtype)
    assert torch.equal(got[1], v)
    # every other place is what it was, bit by bit
    for pool, old in zip(B.cache.pools, before):
        for b, (t, n) in enumerate(zip(lens, new)):
            for pos in range(t - n, t):
                page_id = int(B.table[b, pos // page])
                old[page_id, :, pos % page] = pool[page_id, :, pos % page]
        assert torch.equal(pool.view(torch.int16), old.view(torch.int16))


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_append_without_rotation_strided_and_in_place(dtype):
    lens = [40, 3]
    B = Batch(lens, 2, 128, 16, DTYPES[dtype], seed=5)
    fused = torch.from_numpy(B.rng.standard_normal((43, 12, 128))).to(B.dev, B.dtype)             # 8 + 2 + 2 heads of a row
    q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
    starts, want = B.starts(lens), fused.clone()
    ck.cocktail_kv16_append(B.cache, k, v, starts)
    for b in range(2):
        assert torch.equal(B.pool_rows(b, 0, lens[b], B.cache.k), k[B.rows(b)]) and torch.equal(B.pool_rows(b, 0, lens[b], B.cache.v), v[B.rows(b)])
    rot = _rotation(64)
    out = ck.cocktail_kv16_append(B.cache, k, v, starts, rot, q=q)
    assert torch.equal(fused, want)
    own = q.contiguous()
    assert ck.cocktail_kv16_append(B.cache, k, v, starts, rot, q=own, q_out=own) is own and torch.equal(own, out)
    positions = torch.from_numpy(np.arange(43)[::-1].copy().astype(np.int32)).to(B.dev) * 1000 - 7
    out = ck.cocktail_kv16_append(B.cache, k, v, starts, rot, q=q, positions=positions)
    _check_turned(out, q, positions.cpu().numpy(), _freq(64), False, 1.0, B.dtype)
    got = torch.cat([B.pool_rows(b, 0, lens[b], B.cache.k) for b in range(2)])
    _check_turned(got, k, positions.cpu().numpy(), _freq(64), False, 1.0, B.dtype)
    # heads behind tokens
    k2, v2, q2 = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v, q))
    assert torch.equal(ck.cocktail_kv16_append(B.cache, k2, v2, starts, rot, q=q2, positions=positions), out)


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_at_far_positions(interleaved):
    """Positions up to the ends of 32 bits, where an angle in binary32 would be worth nothing."""
    B = Batch([8], 1, 64, 16, torch.float16, seed=6)
    positions = torch.tensor([0, 1, -1, 131071, 16777217, 2 ** 31 - 1, -2 ** 31, 1999999999], dtype=torch.int32, device=B.dev)
    q = B.query([8], 2)
    out = ck.cocktail_kv16_append(B.cache, B.k, B.v, B.starts([8]), _rotation(64, interleaved), q=q, positions=positions)
    _check_turned(out, q, positions.cpu().numpy(), _freq(64), interleaved, 1.0, B.dtype)
    _check_turned(B.pool_rows(0, 0, 8, B.cache.k), B.k, positions.cpu().numpy(), _freq(64), interleaved, 1.0, B.dtype)


@gpu
def test_rows_that_have_no_place():
    """Pages that are none, tokens before the first, ranges that are none, a resize that found no room."""
    B = Batch([40, 5, 33], 2, 128, 16, torch.float16, seed=7)
    table = B.table.copy()
    table[0, 1], table[1, 0] = B.pages.num_pages, -1
    B.pages.table.copy_(torch.from_numpy(table))
    new = [40, 9, 33]
    k, v, q = (torch.from_numpy(B.rng.standard_normal((82, n, 128))).to(B.dev, B.dtype) for n in (2, 2, 4))
    before = [p.clone() for p in B.cache.pools]
    rot = _rotation(128)
    out = ck.cocktail_kv16_append(B.cache, k, v, B.starts(new), rot, q=q)
    positions = np.concatenate([np.arange(40), np.arange(-4, 5), np.arange(33)])
    _check_turned(out, q, positions, _freq(128), False, 1.0, B.dtype)
    expect = before[1].clone()
    for b, at, skip in ((0, 0, range(16, 32)), (2, 49, ())):
        for pos in range(B.lens[b]):
            if pos not in skip:
                expect[int(table[b, pos // 16]), :, pos % 16] = v[at + pos]
    assert torch.equal(B.cache.v.view(torch.int16), expect.view(torch.int16))
    for bad, left in (([0, 40, 30, 82], None), ([0, 40, 49, 83], 2), ([-3, 40, 49, 82], 0)):
        for p, old in zip(B.cache.pools, before):
            p.copy_(old)
        res = torch.full_like(q, 7.0)
        ck.cocktail_kv16_append(B.cache, k, v, torch.tensor(bad, dtype=torch.int32, device=B.dev), rot, q=q, q_out=res)
        if left is not None:
            rows = slice(max(0, bad[left]), min(82, bad[left + 1]))
            assert (res[rows] == 7.0).all()
            assert torch.equal(B.pool_rows(2, 0, 33, B.cache.v).view(torch.int16), B.pool_rows(2, 0, 33, before[1]).view(torch.int16) if left == 2 else v[49:].view(torch.int16))
        got = ck.cocktail_kv16_attention(B.cache, q, torch.tensor(bad, dtype=torch.int32, device=B.dev), out=torch.full_like(q, 7.0))[0]
        if left is not None:
            assert (got[rows] == 7.0).all()
    # no room: nothing is stored, the queries are turned
    B.pages.status[0] = 3
    for p, old in zip(B.cache.pools, before):
        p.copy_(old)
    res = ck.cocktail_kv16_append(B.cache, k, v, B.starts(new), rot, q=q)
    assert torch.equal(res, out) and torch.equal(B.cache.v.view(torch.int16), before[1].view(torch.int16))
    torch.cuda.synchronize()


CASES = [
    # lens, new, kv heads, query heads per kv head, D, page
    ([1], [1], 1, 1, 128, 16),
    ([0, 1, 15, 16, 17, 31, 32, 33], [1] * 8, 2, 1, 128, 16),
    ([63, 64, 65, 0, 129, 1000], [1] * 6, 2, 4, 64, 48),
    ([700, 0, 5], [1, 0, 1], 3, 8, 128, 64),
    ([300, 20, 1], [2, 2, 2], 2, 16, 128, 16),               # 32 rows: two operands of queries
    ([300, 20, 1], [3, 3, 3], 2, 5, 64, 32),                 # more queries than keys
    ([1500, 40, 333, 2], [1, 40, 7, 2], 2, 6, 128, 16),      # few and many queries in one call
    ([500, 130], [500, 130], 2, 3, 128, 256),                # prompts
    ([257, 64, 1, 0, 191], [257, 64, 1, 0, 100], 1, 2, 64, 16),
    ([2000], [33], 1, 1, 128, 16),                           # few rows, many keys
    ([900, 3], [1, 1], 1, 64, 128, 16),                      # 64 heads per kv head
    ([3000, 10], [5, 10], 1, 40, 64, 80),                    # the keys of a row are cut
    ([100] * 70, [1] * 70, 1, 2, 128, 16),
    ([5] * 300, [1] * 300, 2, 2, 64, 16),
    ([640, 33, 100, 0, 2000, 7], [1, 2, 3, 4, 4, 1], 2, 16, 128, 32),      # one to four operands in one call
    ([640, 33, 100, 0, 2000, 7], [12, 2, 7, 4, 9, 1], 1, 5, 64, 16),
    ([37 * i % 400 for i in range(90)], [1 + i % 3 for i in range(90)], 1, 16, 128, 16),
    ([150 + i % 7 for i in range(80)], [i % 80 for i in range(80)], 1, 2, 128, 16),         # prompts among many sequences
    ([4100, 4096], [70, 65], 2, 2, 64, 64),
    ([1100, 700], [512, 300], 4, 32, 128, 48),               # many rows
    ([1100, 700], [514, 300], 4, 8, 64, 16),
    ([9000, 20], [1, 1], 2, 3, 128, 16),
]


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, dtype):
    lens, new, h, rep, d, page = CASES[case]
    B = Batch(lens, h, d, page, DTYPES[dtype], seed=case, spread=4.0)
    B.store_all()
    q = B.query(new, rep)
    uniform = len(set(new)) == 1
    calls = [dict(starts=B.starts(new))]
    if uniform:
        calls.append(dict())
    calls.append(dict(starts=B.starts(new), max_new=max(new), max_len=max(lens)))
    calls.append(dict(starts=B.starts(new), max_new=max(new), max_len=1))       # a bad guess
    for more in calls:
        out, lse = ck.cocktail_kv16_attention(B.cache, q, **more)
        B.check(q, new, out, lse)
        again, lse2 = ck.cocktail_kv16_attention(B.cache, q, **more)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert torch.equal(B.pages.status.cpu(), torch.zeros(4, dtype=torch.int32))


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("q_scale,kv_scale,sm_scale", [(30.0, 1.0, None), (1e-3, 1.0, None), (1.0, 100.0, 0.02), (0.0, 1.0, None), (1.0, 1e-3, None)])
def test_attention_of_large_and_small_values(new, q_scale, kv_scale, sm_scale, dtype):
    B = Batch([700, 90], 2, 128, 32, DTYPES[dtype], seed=17)
    B.k, B.v = (B.k * kv_scale).to(B.dtype), (B.v * kv_scale).to(B.dtype)
    B.store_all()
    q = B.query([new, new], 4, q_scale)
    out, lse = ck.cocktail_kv16_attention(B.cache, q, sm_scale=sm_scale or 0.0)
    B.check(q, [new, new], out, lse, sm_scale)


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("new", [1, 50])
def test_attention_leaves_out_keys_of_bad_pages(new, dtype):
    B = Batch([200, 77], 2, 64, 16, DTYPES[dtype], seed=18)
    B.store_all()
    table = B.table.copy()
    table[0, [0, 3, 7]] = [-1, 1 << 30, -(1 << 31)]
    table[1, :] = -1
    B.pages.table.copy_(torch.from_numpy(table))
    keep = [np.ones(200, bool), np.zeros(77, bool)]
    for col in (0, 3, 7):
        keep[0][16 * col:16 * col + 16] = False
    q = B.query([new, new], 3)
    out, lse = ck.cocktail_kv16_attention(B.cache, q)
    B.check(q, [new, new], out, lse, keep=keep)


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,new,rep", [([300, 120], [1, 1], 4), ([5000, 120], [3, 2], 16), ([400, 399], [100, 64], 3)])
def test_values_that_are_not_finite_stay_in_their_rows(lens, new, rep, dtype):
    """A query that is NaN or infinite spoils its own rows, a key that is one the rows that see it, a value that is one its channel in its sequence and
    kv head; no others."""
    B = Batch(lens, 2, 128, 16, DTYPES[dtype], seed=19)
    B.store_all()
    q = B.query(new, rep)
    want, wlse = ck.cocktail_kv16_attention(B.cache, q, B.starts(new), max_new=max(new))
    bad = q.clone()
    bad[0, 0, 5], bad[new[0], 1, 0] = float("nan"), float("inf")
    got, lse = ck.cocktail_kv16_attention(B.cache, bad, B.starts(new), max_new=max(new))
    same = torch.ones(q.shape[:2], dtype=torch.bool, device=B.dev)
    same[0, 0] = same[new[0], 1] = False
    assert torch.equal(got[same], want[same]) and torch.equal(lse[same], wlse[same])
    assert got[0, 0].isnan().all() and got[new[0], 1].isnan().all()
    # the last token of the first sequence: only its last query sees it
    t = lens[0] - 1
    page = int(B.table[0, t // 16])
    B.cache.v[page, 1, t % 16, 3] = float("nan")
    B.cache.k[page, 0, t % 16, 3] = float("nan")
    got, lse = ck.cocktail_kv16_attention(B.cache, q, B.starts(new), max_new=max(new))
    last = new[0] - 1
    assert got[last, :rep].isnan().all() and got[last, rep:, 3].isnan().all()
    same = torch.ones(q.shape, dtype=torch.bool, device=B.dev)
    same[last, :rep] = False
    same[:new[0], rep:, 3] = False
    assert torch.equal(got[same], want[same])
    same = torch.ones(q.shape[:2], dtype=torch.bool, device=B.dev)
    same[last, :rep] = False
    assert torch.equal(lse[same], wlse[same])
