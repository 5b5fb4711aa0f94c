"""The paged 4-bit cache: page bookkeeping, store, gather and attention against the oracle in binary64."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck
from oracle import fp4_oracle as O
from paper_2503_23294_amd import _lib

gpu = pytest.mark.gpu
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ---- without a GPU: the oracle against facts of its own, and every refusal of the C entry points ---------------------------------


def test_quantizer_of_the_oracle():
    x = np.zeros(32)
    x[:9] = [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5.5]
    codes, scale = O.quantize(x)
    assert scale[0] == 127 and list(codes[:9]) == [7, 6, 6, 4, 4, 2, 2, 0, 15]          # ties to the even number, 5.5 -> 6
    assert O.quantize(np.zeros(32))[1][0] == 127 - 23
    assert O.quantize(np.full(32, 7.9))[1][0] == 127 and O.value(np.full(32, 7.9))[0] == 6.0       # saturates within the binade
    assert O.value(np.full(32, 1e9))[0] == 49152.0 and O.value(np.full(32, np.inf))[0] == 49152.0
    assert O.value(np.full(32, 2.0 ** -24))[0] == 2.0 ** -24 and O.value(np.full(32, np.nan))[0] == 0.0
    rng = np.random.default_rng(1)
    y = rng.standard_normal((50, 128)) * 10.0 ** rng.uniform(-4, 4, (50, 1))
    v = O.value(y)
    # half a step of the coarsest binade, or what saturates (up to a quarter of the largest value)
    top = np.repeat(np.abs(y).reshape(50, 4, 32).max(axis=-1), 32, axis=1).reshape(50, 128)
    assert (np.abs(v - y) <= top / 4 + 2.0 ** -25).all()
    assert (O.value(v) == v).all()                                                      # values that can be stored are stored
    assert (v.astype(np.float16).astype(np.float64) == v).all()


def test_layout_of_the_oracle_uses_every_byte_once():
    for d, ps in ((64, 16), (128, 48)):
        pool = np.zeros((1, 2 * O.run_bytes(d, ps)), np.uint8)
        seen = np.zeros(pool.shape[1], int)
        rng = np.random.default_rng(0)
        for head in range(2):
            for at in range(ps):
                before = pool.copy()
                k, v = rng.choice([-6.0, 6.0, -4.0], (2, d))                            # no zero bytes
                O.put(pool, 0, at, head, d, ps, k, v)
                seen += (pool != before)[0]
                kk, vv = O.get(pool, 0, at, head, d, ps)
                assert (kk == k).all() and (vv == v).all()
        assert (seen == 1).all()


def _desc(**more):
    d = dict(table=4096, seq_lens=4096, refs=4096, status=4096, num_seqs=4, table_stride=8, page_size=16, num_pages=32)
    d.update(more)
    return _lib.PageTableDesc(*d.values())


def _cache_desc(pool=4096, heads=2, head_dim=128, **more):
    return _lib.Fp4CacheDesc(_desc(**more), pool, heads, head_dim)


@pytest.mark.parametrize("bad,code", [
    (dict(table=None), _lib.EINVAL), (dict(refs=None), _lib.EINVAL), (dict(status=None), _lib.EINVAL), (dict(seq_lens=None), _lib.EINVAL),
    (dict(num_seqs=0), _lib.EINVAL), (dict(num_seqs=4097), _lib.EINVAL), (dict(table_stride=0), _lib.EINVAL), (dict(page_size=0), _lib.EINVAL),
    (dict(num_pages=0), _lib.EINVAL), (dict(num_pages=(1 << 30) + 1), _lib.EINVAL), (dict(table_stride=1 << 27, page_size=16), _lib.EINVAL),
    (dict(table=4098), _lib.EALIGN), (dict(status=4097), _lib.EALIGN)])
def test_page_tables_that_are_refused(bad, code):
    L, d = _lib.lib(), _desc(**bad)
    n = C.c_size_t(0)
    assert L.cocktail_pages_workspace(C.byref(d), C.byref(n)) == code
    assert L.cocktail_pages_fork(C.byref(d), 4096, None) == code
    assert L.cocktail_pages_resize(C.byref(d), 4096, None, 0, 0, 4096, 1 << 20, None) == code
    assert L.cocktail_pages_compact(C.byref(d), None, 0, 0, 4096, 1 << 20, None) == code
    assert L.cocktail_pages_check(C.byref(d), None) == code
    assert L.cocktail_last_error()


def test_refusals_of_the_page_calls():
    L, d = _lib.lib(), _desc()
    n = C.c_size_t(0)
    assert L.cocktail_pages_workspace(C.byref(d), C.byref(n)) == 0 and n.value > 0
    assert L.cocktail_pages_workspace(C.byref(d), None) == _lib.EINVAL and L.cocktail_pages_workspace(None, C.byref(n)) == _lib.EINVAL
    pool = (C.c_void_p * 2)(4096, 8192)
    resize = lambda delta=4096, p=pool, num=2, size=64, ws=4096, wb=n.value: L.cocktail_pages_resize(C.byref(d), delta, p, num, size, ws, wb, None)  # noqa: E731
    assert resize(delta=None) == _lib.EINVAL and resize(delta=2) == _lib.EALIGN
    assert resize(p=None) == _lib.EINVAL and resize(num=-1) == _lib.EINVAL and resize(num=257) == _lib.EINVAL
    assert resize(size=0) == _lib.EINVAL and resize(size=24) == _lib.EINVAL
    assert resize(ws=None) == _lib.EINVAL and resize(ws=8) == _lib.EALIGN and resize(wb=n.value - 1) == _lib.ENOSPACE
    assert resize(p=(C.c_void_p * 2)(4096, None)) == _lib.EINVAL and resize(p=(C.c_void_p * 2)(4096, 8)) == _lib.EALIGN
    assert L.cocktail_pages_compact(C.byref(d), pool, 2, 64, 4096, n.value - 1, None) == _lib.ENOSPACE
    assert L.cocktail_pages_fork(C.byref(d), None, None) == _lib.EINVAL and L.cocktail_pages_fork(C.byref(d), 6, None) == _lib.EALIGN


def test_refusals_of_the_cache_calls():
    L = _lib.lib()
    n = C.c_int64(0)
    assert L.cocktail_fp4_page_bytes(8, 128, 64, C.byref(n)) == 0 and n.value == 8 * 64 * 136
    assert L.cocktail_fp4_page_bytes(3, 64, 16, C.byref(n)) == 0 and n.value == 3 * 16 * 68
    assert L.cocktail_fp4_page_bytes(8, 96, 64, C.byref(n)) == _lib.EUNSUPPORTED
    for args in ((0, 128, 64), (1025, 128, 64), (8, 128, 0), (8, 128, 24), (8, 128, 1 << 17)):
        assert L.cocktail_fp4_page_bytes(*args, C.byref(n)) == _lib.EINVAL, args
    for fn in (L.cocktail_fp4_store, L.cocktail_fp4_gather):
        def call(c=None, k=4096, v=4096, dtype=0, st=256, sh=128, total=8, starts=4096):
            return fn(C.byref(c or _cache_desc()), k, v, dtype, st, sh, total, starts, None)
        assert fn(None, 4096, 4096, 0, 256, 128, 8, None, None) == _lib.EINVAL
        assert call(c=_cache_desc(head_dim=80)) == _lib.EUNSUPPORTED and call(c=_cache_desc(pool=None)) == _lib.EINVAL
        assert call(c=_cache_desc(pool=8)) == _lib.EALIGN and call(c=_cache_desc(page_size=8)) == _lib.EINVAL
        assert call(k=None) == _lib.EINVAL and call(v=None) == _lib.EINVAL and call(k=8) == _lib.EALIGN and call(dtype=2) == _lib.EINVAL
        assert call(st=130) == _lib.EINVAL and call(st=-256) == _lib.EINVAL and call(sh=4) == _lib.EINVAL
        assert call(st=120) == _lib.EINVAL and call(sh=64) == _lib.EINVAL                # rows or heads on top of each other
        assert call(total=-1) == _lib.EINVAL and call(starts=2) == _lib.EALIGN
        assert call(total=6, starts=None) == _lib.EINVAL                                 # four sequences
        assert call(total=0) == 0                                                        # nothing to do: nothing is launched


def test_refusals_of_attention():
    L = _lib.lib()
    n = C.c_size_t(0)

    def call(c=None, hq=4, q=4096, dtype=0, st=512, sh=128, total=8, starts=4096, max_new=8, max_len=0, scale=0.0, out=4096, lse=None, ws=4096, wb=1 << 40):
        return L.cocktail_fp4_attention(C.byref(c or _cache_desc()), hq, q, dtype, st, sh, total, starts, max_new, max_len, scale, out, lse, ws, wb, None)
    assert L.cocktail_fp4_attention_workspace(C.byref(_cache_desc()), 4, 8, 8, 0, 0, C.byref(n)) == 0 and n.value > 0
    assert L.cocktail_fp4_attention_workspace(C.byref(_cache_desc()), 4, 8, 8, 0, 0, None) == _lib.EINVAL
    assert call(wb=n.value - 1) == _lib.ENOSPACE
    assert call(hq=3) == _lib.EINVAL and call(hq=0) == _lib.EINVAL and call(hq=130) == _lib.EUNSUPPORTED
    assert call(q=None) == _lib.EINVAL and call(out=None) == _lib.EINVAL and call(q=4104) == _lib.EALIGN and call(dtype=7) == _lib.EINVAL
    assert call(max_new=0) == _lib.EINVAL and call(max_new=9) == _lib.EINVAL and call(total=-1) == _lib.EINVAL
    assert call(starts=None, max_new=3) == _lib.EINVAL and call(total=6, starts=None, max_new=1) == _lib.EINVAL
    assert call(scale=float("nan")) == _lib.EINVAL and call(scale=float("inf")) == _lib.EINVAL
    assert call(ws=None) == _lib.EINVAL and call(ws=8) == _lib.EALIGN and call(lse=2) == _lib.EALIGN
    assert call(c=_cache_desc(head_dim=32)) == _lib.EUNSUPPORTED
    assert call(c=_cache_desc(num_seqs=4096, table_stride=1 << 26, page_size=16)) == _lib.EINVAL   # more units than are numbered
    assert call(total=0, max_new=0) == 0


def test_refusals_of_what_32_bits_do_not_number():
    """Positions near 2^31, and launches of 2^32 threads."""
    L = _lib.lib()
    n = C.c_size_t(0)
    far, near = _cache_desc(table_stride=(1 << 27) - 1), _cache_desc(num_seqs=1, table_stride=(1 << 27) - 16)
    assert L.cocktail_fp4_store(C.byref(far), 4096, 4096, 0, 256, 128, 8, 4096, None) == _lib.EINVAL
    assert L.cocktail_fp4_gather(C.byref(far), 4096, 4096, 0, 256, 128, 8, 4096, None) == _lib.EINVAL
    assert L.cocktail_fp4_attention_workspace(C.byref(far), 4, 8, 8, 0, 0, C.byref(n)) == _lib.EINVAL
    assert L.cocktail_fp4_attention_workspace(C.byref(near), 4, 8, 8, 0, 0, C.byref(n)) == 0
    wide = _cache_desc(heads=512)
    for fn in (L.cocktail_fp4_store, L.cocktail_fp4_gather):
        assert fn(C.byref(wide), 4096, 4096, 0, 512 * 128, 128, 1 << 22, 4096, None) == _lib.EINVAL   # 2^20 quads of 2^14 threads
        assert b"more than one launch" in L.cocktail_last_error()


def test_the_binding_wants_device_tensors():
    with pytest.raises(TypeError):
        ck.PageTable(2, 64, 8, 16, torch.device("cpu"))


# ---- on the GPU ------------------------------------------------------------------------------------------------------------


def _f64(t):
    return t.detach().cpu().double().numpy()


class Batch:
    """A cache whose pages lie in random places of a pool full of junk (scales that mean NaN among it), with the source it holds."""

    def __init__(self, lens, kv_heads, head_dim, page, dtype, seed=0, spread=1.0, spare=3):
        self.dev = torch.device("cuda:0")
        self.lens, self.h, self.d, self.page, self.dtype = list(lens), kv_heads, head_dim, page, dtype
        rng = np.random.default_rng(seed)
        need = [-(-t // page) for t in lens]
        pages = sum(need) + spare
        ids = rng.permutation(pages).astype(np.int32)
        # room for long contexts, so that calls that name no length are cut as for those
        table = np.full((len(lens), max(max(need) + 1, 20000 // page)), -1, np.int32)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = ids[at:at + k]
            at += k
        refs = np.zeros(pages, np.int32)
        refs[ids[:at]] = 1
        t = lambda a: torch.from_numpy(a).to(self.dev)  # noqa: E731
        self.pages = ck.PageTable.of(t(table), t(np.array(lens, np.int32)), t(refs), page)
        self.cache = ck.Fp4Cache(self.pages, kv_heads, head_dim)
        self.junk = rng.integers(0, 256, tuple(self.cache.pool.shape), dtype=np.uint8)
        self.junk[rng.random(self.junk.shape) < 0.3] = 255
        self.cache.pool.copy_(t(self.junk))
        make = lambda: torch.from_numpy(rng.standard_normal((sum(lens), kv_heads, head_dim)) * spread ** rng.uniform(-1, 1, (sum(lens), kv_heads, 1))).to(self.dev, dtype)  # noqa: E731
        self.k, self.v = make(), make()
        self.rng = rng

    def starts(self, counts):
        return torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(self.dev)

    def store_all(self):
        ck.cocktail_fp4_store(self.cache, self.k, self.v, self.starts(self.lens))

    def rows(self, b):
        at = sum(self.lens[:b])
        return slice(at, at + self.lens[b])

    def query(self, new, rep, scale=1.0):
        return torch.from_numpy(self.rng.standard_normal((sum(new), self.h * rep, self.d)) * scale).to(self.dev, self.dtype)

    def check(self, q, new, out, lse, sm_scale=None, keep=None):
        """Against binary64.  Bounds: the result's own rounding (half a step); weights rounded to fp16, in the sum over V and in the normaliser (2^-11
        each at most), and, where they are fp16 subnormals, by 2^-25 of the reference; logits: D products and sums in binary32 of terms whose
        magnitudes sum to `size`, and the smallest channels of a bf16 query; sums over the keys in binary32."""
        eps = torch.finfo(q.dtype).eps / 2
        qd, kd, vd, od, ld = _f64(q), O.value(_f64(self.k)), O.value(_f64(self.v)), _f64(out), _f64(lse)
        at = 0
        for b, n in enumerate(new):
            if not n:
                continue
            t, r = self.lens[b], self.rows(b)
            kb, vb, qb = kd[r], vd[r], qd[at:at + n]
            pad = max(0, n - t)      # queries before the first token
            want, wl, mean_v, size = O.attention(qb[pad:], kb, vb, None if keep is None else keep[b], sm_scale)
            got, gl = od[at:at + n], ld[at:at + n]
            assert (got[:pad] == 0).all() and np.isneginf(gl[:pad]).all(), f"sequence {b}: queries without keys"
            got, gl = got[pad:], gl[pad:]
            none = np.isneginf(wl)
            assert (got[none] == 0).all() and (np.isneginf(gl) == none).all(), f"sequence {b}: rows without keys"
            logit = (self.d + 4) * 2.0 ** -24 * size + 2.0 ** -21 * (1 + np.abs(np.where(none, 0, wl))) + 2.0 ** -20
            if q.dtype == torch.bfloat16:
                scale = sm_scale or 1 / math.sqrt(self.d)
                logit = logit + 2.0 ** -24 * scale * np.abs(qb[pad:]).max(-1) * (np.abs(kb).sum(-1).max() if t else 0)
            weight = 2 * (2.0 ** -11 + logit + t * 2.0 ** -24)
            bound = eps * np.abs(want) + weight[..., None] * mean_v * (1 + eps) + t * 2.0 ** -25 * (np.abs(vb).max() if t else 0) + 2.0 ** -25
            far = np.abs(got - want)
            assert (far <= bound).all(), f"sequence {b}: {np.max(far - bound)} over, {np.max(far)} off, at {np.argwhere(far > bound)[:4].tolist()}"
            far = np.abs(np.where(none, 0, gl) - np.where(none, 0, wl))
            assert (far <= logit + t * 2.0 ** -24).all(), f"sequence {b}: lse off by {far.max()}"
            at += n


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,d,page", [(2, 128, 16), (3, 64, 48), (1, 128, 64), (5, 64, 16)])
def test_store_writes_the_layout_and_nothing_else(heads, d, page, dtype):
    """All tokens at once, then new ones on top that begin and end inside quads: byte for byte."""
    lens = [37, 0, 1, 64, 18]
    B = Batch(lens, heads, d, page, DTYPES[dtype], seed=heads + d, spread=30.0)
    with torch.no_grad():
        flat = B.k.view(-1)
        special = torch.tensor([0.0, -0.0, float("inf"), -float("inf"), float("nan"), 6e4, 6e-8, -1e-7, 5.0, 3.5], device=B.dev, dtype=B.dtype)
        flat[:10] = special
        B.k[3, 0] = 0.0
        B.k[4, 0, :32] = torch.tensor([-0.0] * 31 + [1.0], device=B.dev, dtype=B.dtype)
        B.v[5, 0, 32:64] = 2.0 ** -24
        B.v[6, 0, 0] = float("nan")
        if dtype == "bf16":
            B.v[7, 0, 0] = 3e38
    counts = [30, 0, 1, 7, 18]                                # the last ones of every sequence
    parts = [B.rows(b) for b in range(5)]
    new = torch.cat([torch.arange(p.stop - n, p.stop) for p, n in zip(parts, counts)])
    # rows of a fused projection: strides of their own
    wide = torch.randn(len(new), 3 * heads * d + 8, device=B.dev).to(B.dtype)
    ks, vs = (wide[:, i * heads * d:(i + 1) * heads * d].unflatten(1, (heads, d)) for i in range(2))
    ks.copy_(B.k[new.to(B.dev)])
    vs.copy_(B.v[new.to(B.dev)])
    want = B.junk.copy()
    table, kd, vd = B.pages.table.cpu().numpy(), _f64(B.k), _f64(B.v)

    def put(b, tokens):
        for t in tokens:
            for h in range(heads):
                row = parts[b].start + t
                O.put(want, table[b, t // page], t % page, h, d, page, kd[row, h], vd[row, h])
    ck.cocktail_fp4_store(B.cache, ks, vs, B.starts(counts))
    for b, n in enumerate(counts):
        put(b, range(lens[b] - n, lens[b]))
    assert np.array_equal(B.cache.pool.cpu().numpy(), want)
    B.store_all()
    for b in range(5):
        put(b, range(lens[b]))
    assert np.array_equal(B.cache.pool.cpu().numpy(), want)
    for out_type in (torch.float16, torch.bfloat16):
        k, v = ck.cocktail_fp4_gather(B.cache, sum(counts), B.starts(counts), dtype=out_type)
        assert np.array_equal(_f64(k), O.value(kd[new])) and np.array_equal(_f64(v), O.value(vd[new]))


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_store_and_gather_every_value(dtype):
    """All 65536 bit patterns, in groups whose largest value varies."""
    bits = np.arange(65536, dtype=np.uint16)
    bits = np.concatenate([bits, np.random.default_rng(3).permutation(bits)]).view(np.int16)
    x = torch.from_numpy(bits).view(DTYPES[dtype]).view(-1, 2, 64).cuda()
    B = Batch([x.shape[0]], 2, 64, 64, DTYPES[dtype])
    B.k, B.v = x, x.flip(0).contiguous()
    B.store_all()
    k, v = ck.cocktail_fp4_gather(B.cache, x.shape[0], dtype=DTYPES[dtype])
    assert np.array_equal(_f64(k), O.value(_f64(x))) and np.array_equal(_f64(v), O.value(_f64(B.v)))


@gpu
def test_rows_that_have_no_place():
    """Rows before the first token, on pages that are none, of ranges that are none: left out, read as zeros or not written."""
    B = Batch([40, 20, 33], 2, 128, 16, torch.float16, seed=5)
    pool = B.cache.pool.clone()
    table = B.pages.table.clone()
    B.pages.table[0, 1], B.pages.table[1, 0] = B.pages.num_pages, -5
    counts = [40, 25, 33]
    x = torch.randn(sum(counts), 2, 128, device=B.dev).half()
    ck.cocktail_fp4_store(B.cache, x, x, B.starts(counts))
    k, v = ck.cocktail_fp4_gather(B.cache, sum(counts), B.starts(counts))
    kd, want = _f64(k), O.value(_f64(x))
    want[16:32] = 0                      # second page of sequence 0
    want[40:40 + 5 + 16] = 0             # before its first token, and the first page
    assert np.array_equal(kd, want) and np.array_equal(_f64(v), want)
    used = set(table[0, [0, 2]].tolist() + table[1, [1]].tolist() + table[2, :3].tolist())
    same = [i for i in range(B.pages.num_pages) if i not in used]
    assert torch.equal(B.cache.pool[same], pool[same])
    # a range that goes backwards, one that leaves the batch, one before it
    for bad in ([0, 40, 30, 98], [0, 40, 65, 99], [-3, 40, 65, 98]):
        B.cache.pool.copy_(pool)
        out = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
        starts = torch.tensor(bad, dtype=torch.int32, device=B.dev)
        ck.cocktail_fp4_store(B.cache, x, x, starts)
        ck.cocktail_fp4_gather(B.cache, 98, starts, out=out)
        left = 1 if bad[2] == 30 else 2 if bad[3] == 99 else 0
        rows = slice(max(0, bad[left]), min(98, max(bad[left:left + 2])))
        if left != 1:
            assert (out[0][rows] == 7.0).all()
        q = torch.randn(98, 4, 128, device=B.dev).half()
        res = torch.full_like(q, 7.0)
        ck.cocktail_fp4_attention(B.cache, q, starts, out=res)
        if left != 1:
            assert (res[rows] == 7.0).all()
    torch.cuda.synchronize()


CASES = [
    # lens, new, kv heads, query heads per kv head, D, page
    ([1], [1], 1, 1, 128, 16),
    ([0, 1, 15, 16, 17, 31, 32, 33], [1] * 8, 2, 1, 128, 16),
    ([63, 64, 65, 0, 129, 1000], [1] * 6, 2, 4, 64, 48),
    ([700, 0, 5], [1, 0, 1], 3, 8, 128, 64),
    ([300, 20, 1], [2, 2, 2], 2, 16, 128, 16),               # 32 rows: two operands of queries
    ([300, 20, 1], [3, 3, 3], 2, 5, 64, 32),                 # more queries than keys
    ([1500, 40, 333, 2], [1, 40, 7, 2], 2, 6, 128, 16),      # both kernels in one call
    ([500, 130], [500, 130], 2, 3, 128, 256),                # prompts
    ([257, 64, 1, 0, 191], [257, 64, 1, 0, 100], 1, 2, 64, 16),
    ([2000], [33], 1, 1, 128, 16),                           # few rows, many keys
    ([900, 3], [1, 1], 1, 64, 128, 16),                      # 64 heads per kv head
    ([3000, 10], [5, 10], 1, 40, 64, 80),                    # the keys of a row are cut
    ([100] * 70, [1] * 70, 1, 2, 128, 16),
    ([5] * 300, [1] * 300, 2, 2, 64, 16),
    ([640, 33, 100, 0, 2000, 7], [1, 2, 3, 4, 4, 1], 2, 16, 128, 32),      # one to four operands in one call
    ([640, 33, 100, 0, 2000, 7], [12, 2, 7, 4, 9, 1], 1, 5, 64, 16),
    ([37 * i % 400 for i in range(90)], [1 + i % 3 for i in range(90)], 1, 16, 128, 16),   # the same, found in shared memory
    ([150 + i % 7 for i in range(80)], [i % 80 for i in range(80)], 1, 2, 128, 16),         # prompts among many sequences
    ([4100, 4096], [70, 65], 2, 2, 64, 64),
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
        out, lse = ck.cocktail_fp4_attention(B.cache, q, **more)
        B.check(q, new, out, lse)
        again, lse2 = ck.cocktail_fp4_attention(B.cache, q, **more)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert torch.equal(B.pages.status.cpu(), torch.zeros(4, dtype=torch.int32))


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,rep", [([1100, 700], [512, 300], 32), ([700, 333], [700, 333], 24)])
def test_attention_of_many_rows(lens, new, rep, d):
    """Enough rows for workgroups of eight waves, and of four without cut keys."""
    B = Batch(lens, 4, d, 48, torch.float16, seed=d, spread=2.0)
    B.store_all()
    q = B.query(new, rep)
    out, lse = ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=max(new), max_len=max(lens))
    B.check(q, new, out, lse)


@gpu
@pytest.mark.parametrize("num_seqs", [70, 1500, 4096])
def test_few_active_sequences_in_a_large_table(num_seqs):
    """A table with room for many sequences, of which a few generate: one of them has no key, one many queries."""
    rng = np.random.default_rng(num_seqs)
    active = np.sort(rng.choice(num_seqs, 6, replace=False))
    lens, new = np.zeros(num_seqs, int), np.zeros(num_seqs, int)
    lens[active], new[active] = [300, 0, 77, 1000, 16, 130], [1, 1, 2, 1, 1, 1]
    for most in (2, 60):
        new[active[-1]] = most - 1
        B = Batch(lens.tolist(), 2, 64, 16, torch.float16, seed=num_seqs)
        B.store_all()
        q = B.query(new.tolist(), 4)
        for max_len in (1000, 0):
            out, lse = ck.cocktail_fp4_attention(B.cache, q, B.starts(new.tolist()), max_new=most, max_len=max_len)
            B.check(q, new.tolist(), out, lse)


@gpu
def test_prompts_alone():
    """No sequence can have few queries by the sizes of the call, so one kernel has them all: also a sequence that has few, next to one that has more than
    it may and is left out."""
    B = Batch([400, 390], 2, 128, 16, torch.float16, seed=41)
    B.store_all()
    for new in ([200, 100], [200, 200], [150, 130]):
        q = B.query(new, 3)
        out, lse = ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=200, max_len=400)
        B.check(q, new, out, lse)
    new = [295, 5]
    q = B.query(new, 3)
    out, lse = torch.full_like(q, 7.0), torch.full((300, 6), 7.0, device=B.dev)
    ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=200, max_len=400, out=out, lse=lse)
    assert (out[:295] == 7.0).all() and (lse[:295] == 7.0).all()
    B.check(q[295:], [0, 5], out[295:], lse[295:])


@gpu
@pytest.mark.parametrize("num_seqs,heads", [(40, 8), (64, 9), (33, 31), (64, 4), (65, 8)])
def test_many_segments_of_unlike_lengths(num_seqs, heads):
    """More short segments than compute units, in the order of their lengths: lengths that are alike or zero, sequences without queries."""
    rng = np.random.default_rng(num_seqs)
    lens = rng.choice([0, 1, 31, 32, 33, 64, 100, 257, 700], num_seqs)
    new = (rng.random(num_seqs) < 0.8).astype(int)
    new[lens == 0] = [1 - i % 2 for i in range(int((lens == 0).sum()))]
    B = Batch(lens.tolist(), heads, 64, 32, torch.bfloat16, seed=heads)
    B.store_all()
    q = B.query(new.tolist(), 2)
    out, lse = ck.cocktail_fp4_attention(B.cache, q, B.starts(new.tolist()), max_new=1, max_len=700)
    B.check(q, new.tolist(), out, lse)


@gpu
@pytest.mark.parametrize("new", [1, 3, 100])
def test_attention_over_a_cache_beyond_the_last_cache(new):
    """285 MB of keys and values: read past the caches where a row's keys are read once.  Reference in binary64 on the device, from the cache's own
    values (what they are is the store's test)."""
    dev, t, h, d, rep = torch.device("cuda:0"), 262144 + 17, 8, 128, 4
    pages = ck.PageTable(1, t, -(-t // 64), 64, dev)
    cache = ck.Fp4Cache(pages, h, d)
    ck.cocktail_pages_resize(pages, torch.tensor([t], dtype=torch.int32).to(dev))
    k, v = (torch.randn(t, h, d, device=dev, dtype=torch.float16) for _ in range(2))
    ck.cocktail_fp4_store(cache, k, v)
    k, v = ck.cocktail_fp4_gather(cache, t)
    q = torch.randn(new, h * rep, d, device=dev, dtype=torch.float16)
    q[:, 0] = 3 * k[t // 2, 0]                        # a row that looks at one key
    out, lse = ck.cocktail_fp4_attention(cache, q)
    for i in range(h * rep):
        kk, vv = k[:, i // rep].double(), v[:, i // rep].double()
        s = q[:, i].double() @ kk.t() / math.sqrt(d)
        s.masked_fill_(torch.arange(t, device=dev)[None] > torch.arange(t - new, t, device=dev)[:, None], -math.inf)
        w = torch.softmax(s, dim=1)
        want, mean_v = w @ vv, w @ vv.abs()
        # the result's rounding; the weights', in the sum over V and in the normaliser (2^-11 each), with logits of up to 40 in size, whose products and
        # sums in binary32 are off by 132 * 2^-24 * 40 = 3.2e-4, and sums over the keys in parts of a few thousand; weights that are fp16
        # subnormals: 2^-25 of the largest each, against a sum of `total` largest
        total = torch.exp(torch.logsumexp(s, dim=1) - s.amax(dim=1))
        bound = 2.0 ** -11 * want.abs() + (2.0 ** -10 + 2 * 3.2e-4 + 4096 * 2.0 ** -24) * mean_v + (t * 2.0 ** -25 * vv.abs().max() / total)[:, None]
        assert ((out[:, i].double() - want).abs() <= bound).all(), i
        assert ((lse[:, i].double() - torch.logsumexp(s, dim=1)).abs() <= 3.2e-4 + 4096 * 2.0 ** -24 + 2.0 ** -17).all()


@gpu
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("q_scale,kv_scale,sm_scale", [(30.0, 1.0, None), (1e-6, 1.0, None), (1.0, 300.0, 0.02), (0.0, 1.0, None), (1.0, 1e-5, 50.0), (3.0, 3.0, 1.0)])
def test_attention_of_large_and_small_values(new, q_scale, kv_scale, sm_scale):
    for dtype in DTYPES.values():
        B = Batch([400, 77], 2, 128, 32, dtype, seed=11)
        with torch.no_grad():
            B.k.mul_(kv_scale)
            B.v.mul_(kv_scale)
            B.k[60:].mul_(0.25)          # the largest logits are early, then late ones that raise the maximum
            B.k[390].mul_(8)
        B.store_all()
        q = B.query([new, new], 4, q_scale)
        if q_scale == 3.0:
            q[:, :, ::5] = 2.0 ** -13 * q[:, :, ::5]         # channels of unlike size
        out, lse = ck.cocktail_fp4_attention(B.cache, q, sm_scale=sm_scale or 0.0)
        B.check(q, [new, new], out, lse, sm_scale)


@gpu
@pytest.mark.parametrize("new", [1, 50])
def test_attention_leaves_out_keys_of_bad_pages(new):
    B = Batch([200, 64, 48], 2, 128, 16, torch.float16, seed=3)
    B.store_all()
    keep = [np.ones(t, bool) for t in B.lens]
    for b, col, bad in ((0, 0, -1), (0, 5, B.pages.num_pages), (0, 12, 1 << 30), (1, 1, -2 ** 31), (2, 0, -1), (2, 1, -1), (2, 2, -1)):
        B.pages.table[b, col] = bad
        keep[b][col * 16:(col + 1) * 16] = False
    counts = [new, new, min(new, 48)]
    q = B.query(counts, 2)
    out, lse = ck.cocktail_fp4_attention(B.cache, q, B.starts(counts))
    B.check(q, counts, out, lse, keep=keep)


@gpu
def test_strided_queries_and_rows_of_other_sequences_stay():
    """Queries as a slice of a fused projection; rows behind the last sequence and of sequences with too many queries stay as they were."""
    B = Batch([120, 60, 90], 2, 64, 16, torch.bfloat16, seed=9)
    B.store_all()
    new = [3, 20, 2]
    q = B.query(new, 3)
    wide = torch.randn(30, 6 * 64 * 2 + 16, device=B.dev).to(q.dtype)
    view = wide[:, 8:8 + 6 * 64].unflatten(1, (6, 64))
    view[:25] = q
    out = torch.full((30, 6, 64), 5.0, device=B.dev, dtype=q.dtype)
    lse = torch.full((30, 6), 5.0, device=B.dev)
    ck.cocktail_fp4_attention(B.cache, view, B.starts(new), out=out, lse=lse)
    B.check(q, new, out[:25], lse[:25])
    assert (out[25:] == 5.0).all() and (lse[25:] == 5.0).all()
    out.fill_(5.0)
    ck.cocktail_fp4_attention(B.cache, view, B.starts(new), max_new=4, out=out)
    assert (out[3:23] == 5.0).all() and (out[:3] != 5.0).any()


@gpu
def test_pools_beyond_32_bits():
    """Pages that lie more than 4 GiB into the pool, and codes of K that do within a large page."""
    dev = torch.device("cuda:0")
    for heads, d, page, num_pages in ((8, 128, 64, 70000), (2, 128, 65536, 260)):
        pages = ck.PageTable(2, 4 * page, num_pages, page, dev)
        cache = ck.Fp4Cache(pages, heads, d)
        assert cache.pool.numel() > 1 << 32
        lens = [page + 70, 30]
        pages.table[0, 0], pages.table[0, 1], pages.table[1, 0] = num_pages - 1, num_pages - 2, num_pages // 2 + 3
        pages.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        k, v = (torch.randn(sum(lens), heads, d, device=dev, dtype=torch.float16) for _ in range(2))
        starts = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device=dev)
        ck.cocktail_fp4_store(cache, k, v, starts)
        gk, gv = ck.cocktail_fp4_gather(cache, sum(lens), starts)
        has = 2 * page                                   # tokens of sequence 0 beyond its second page have no place
        tail = np.arange(lens[0] - 200 if page > 100 else 0, sum(lens))
        lost = (tail >= has) & (tail < lens[0])
        idx = torch.from_numpy(tail).to(dev)
        for got, given in ((gk, k), (gv, v)):
            assert np.array_equal(_f64(got[idx]), np.where(lost[:, None, None], 0.0, O.value(_f64(given[idx]))))
        q = torch.randn(2, heads, d, device=dev, dtype=torch.float16)
        out, _ = ck.cocktail_fp4_attention(cache, q)
        for b, rows in enumerate((slice(0, lens[0]), slice(lens[0], None))):
            want, _, mean_v, _ = O.attention(_f64(q[b:b + 1]), _f64(gk[rows]), _f64(gv[rows]), np.arange(lens[b]) < has)
            assert (np.abs(_f64(out[b:b + 1]) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -9 * mean_v).all()
        del cache, pages, k, v, gk, gv
        torch.cuda.empty_cache()


# ---- pages -------------------------------------------------------------------------------------------------------------------


class Twin:
    """A page table on the device and the oracle's, and a pool whose pages hold known contents."""

    def __init__(self, num_seqs, stride, num_pages, page, pools=2, elems=24):
        self.dev = torch.device("cuda:0")
        self.model = O.Pages(num_seqs, stride, num_pages, page)
        self.pages = ck.PageTable(num_seqs, stride * page, num_pages, page, self.dev)
        self.pools = [torch.randint(-2 ** 31, 2 ** 31 - 1, (num_pages, elems), dtype=torch.int32, device=self.dev) for _ in range(pools)]
        self.shadow = [p.cpu().numpy().copy() for p in self.pools]

    def _moved(self, moves):
        for s in self.shadow:
            for a, b in moves:
                s[b] = s[a]

    def resize(self, delta, pools=True):
        ck.cocktail_pages_resize(self.pages, torch.tensor(delta, dtype=torch.int32).to(self.dev), self.pools if pools else [])
        self._moved(self.model.resize(delta, pools))
        self.same()

    def fork(self, source):
        ck.cocktail_pages_fork(self.pages, torch.tensor(source, dtype=torch.int32).to(self.dev))
        self.model.fork(source)
        self.same()

    def compact(self):
        ck.cocktail_pages_compact(self.pages, self.pools)
        self._moved(self.model.compact())
        self.same()

    def same(self):
        assert np.array_equal(self.pages.table.cpu().numpy(), self.model.table())
        assert self.pages.seq_lens.tolist() == self.model.lens and self.pages.refs.tolist() == self.model.refs
        assert self.pages.status.tolist() == [self.model.status, 0, 0, 0]
        for p, s in zip(self.pools, self.shadow):
            assert np.array_equal(p.cpu().numpy(), s)


@gpu
def test_page_operations_one_by_one():
    T = Twin(5, 6, 16, 16)
    T.resize([20, 0, 16, 5, 0])                    # whole and partly filled pages
    T.fork([0, 0, 2, 3, 0])                        # three rows share a partly filled page
    T.resize([1, 1, 1, 0, 0])                      # two of them grow, the third keeps the page: both copy; row 2 takes a new page
    T.resize([0, 0, 0, 0, 1])                      # now it is its own
    T.fork([3, 0, 2, 3, 1])                        # rows change places and are shared at once
    T.resize([3, 0, 0, 3, 0])                      # all holders grow: the last one keeps the page
    T.fork([0, -1, 9, 3, -2 ** 31])                # freed; a source that is no sequence
    T.resize([-7, 30, -2 ** 31, 0, 0])
    T.compact()
    T.compact()                                    # nothing left to do
    T.resize([0, 0, 0, 200, 0])                    # more columns than there are
    assert T.model.status == -1
    with pytest.raises(ck.CocktailError):
        ck.cocktail_pages_check(T.pages)
    T.resize([60, 10, 80, 0, 90])                  # more pages than there are
    assert T.model.status > 0
    with pytest.raises(ck.CocktailError):
        ck.cocktail_pages_check(T.pages)
    T.fork([3, 3, 2, 3, 4])
    T.resize([1, 0, 0, 0, 0], pools=False)         # a copy is due and there are no pools
    assert T.model.status == -2
    with pytest.raises(ck.CocktailError):
        ck.cocktail_pages_check(T.pages)
    T.resize([0, 0, 0, 0, 0])
    ck.cocktail_pages_check(T.pages)
    T.resize([-10 ** 9] * 5)
    assert T.model.refs == [0] * 16


@gpu
@pytest.mark.parametrize("num_seqs,stride,num_pages,page,elems", [(1, 1, 1, 1, 4), (3, 40, 60, 1, 4), (7, 9, 40, 16, 24), (64, 30, 900, 16, 8192),
                                                                  (300, 5, 1100, 7, 4), (1030, 20, 9001, 16, 4)])
def test_page_operations_at_random(num_seqs, stride, num_pages, page, elems):
    rng = np.random.default_rng(num_seqs)
    T = Twin(num_seqs, stride, num_pages, page, pools=1 if elems > 100 else 3, elems=elems)
    most = stride * page
    for step in range(14 if num_seqs < 1000 else 6):
        kind = rng.integers(0, 4)
        if kind <= 1:
            delta = rng.integers(-most // 4, most // 3 + 2, num_seqs) if kind else rng.integers(0, 3, num_seqs)
            delta = np.where(rng.random(num_seqs) < 0.1, -2 ** 31, delta)
            if rng.random() < 0.8:
                delta = np.minimum(delta, most - np.array(T.model.lens))
            T.resize([int(x) for x in delta])
        elif kind == 2:
            src = np.where(rng.random(num_seqs) < 0.6, np.arange(num_seqs), rng.integers(-2, num_seqs + 1, num_seqs))
            T.fork([int(x) for x in src])
        else:
            T.compact()


@gpu
def test_many_pools_and_large_tables():
    """As many pools as a call takes, and as many sequences."""
    T = Twin(4096, 3, 6000, 16, pools=256, elems=4)
    T.resize([17] * 2048 + [0] * 2048)
    T.fork(list(range(2048)) + list(range(2048)))
    T.resize([0] * 2048 + [1] * 1500 + [0] * 548)
    T.fork([-1] * 100 + list(range(100, 4096)))
    T.compact()


# ---- together ------------------------------------------------------------------------------------------------------------------


class Serving:
    """A batch as a program runs it, and next to it what every sequence has been given."""

    def __init__(self, num_seqs, heads, d, page, num_pages, dtype, layers=2, seed=0):
        self.dev = torch.device("cuda:0")
        self.pages = ck.PageTable(num_seqs, 40 * page, num_pages, page, self.dev)
        self.caches = [ck.Fp4Cache(self.pages, heads, d) for _ in range(layers)]
        self.given = [[[] for _ in range(num_seqs)] for _ in range(layers)]
        self.h, self.d, self.dtype, self.n = heads, d, dtype, num_seqs
        self.rng = torch.Generator(device="cuda").manual_seed(seed)

    def pools(self):
        return [c.pool for c in self.caches]

    def randn(self, *shape):
        return torch.randn(*shape, device=self.dev, generator=self.rng).to(self.dtype)

    def step(self, counts, rep=4, check=True):
        """counts[b] new tokens of every sequence: room, store, attend, in every layer."""
        delta = torch.tensor(counts, dtype=torch.int32).to(self.dev)
        starts = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(self.dev)
        ck.cocktail_pages_resize(self.pages, delta, self.pools())
        for layer, cache in enumerate(self.caches):
            k, v = self.randn(sum(counts), self.h, self.d), self.randn(sum(counts), self.h, self.d)
            q = self.randn(sum(counts), self.h * rep, self.d)
            ck.cocktail_fp4_store(cache, k, v, starts)
            out, lse = ck.cocktail_fp4_attention(cache, q, starts)
            at = 0
            for b, c in enumerate(counts):
                self.given[layer][b].extend((k[at + i], v[at + i]) for i in range(c))
                at += c
            if check:
                self.verify(layer, q, counts, out)
        ck.cocktail_pages_check(self.pages)

    def verify(self, layer, q, counts, out):
        at = 0
        for b, n in enumerate(counts):
            if n:
                k, v = (O.value(np.stack([_f64(x[i]) for x in self.given[layer][b]])) for i in range(2))
                want, _, mean_v, _ = O.attention(_f64(q[at:at + n]), k, v)
                eps = torch.finfo(self.dtype).eps / 2
                # the result's rounding and that of the weights, twice; logits of unit normals add less than the slack of 2^-12
                assert (np.abs(_f64(out[at:at + n]) - want) <= eps * np.abs(want) + 2.5 * 2.0 ** -11 * mean_v).all(), (layer, b)
            at += n

    def fork(self, source):
        ck.cocktail_pages_fork(self.pages, torch.tensor(source, dtype=torch.int32).to(self.dev))
        for layer in range(len(self.caches)):
            old = [list(x) for x in self.given[layer]]
            self.given[layer] = [old[s] if s >= 0 else [] for s in source]
            self.given[layer] = [list(x) for x in self.given[layer]]


@gpu
@pytest.mark.parametrize("dtype,d,page", [("fp16", 128, 16), ("bf16", 64, 32)])
def test_a_batch_from_prompts_to_forks_and_back(dtype, d, page):
    S = Serving(5, 2, d, page, 60, DTYPES[dtype])
    S.step([70, 0, 33, 1, 0])                       # prompts
    S.step([1, 17, 1, 1, 0])                        # two more join, the others generate
    S.fork([0, 1, 2, 0, 0])                         # three hypotheses of sequence 0, sequence 3 is gone
    S.step([1, 1, 1, 1, 1])
    S.step([4, 0, 2, 1, 1])                         # drafts
    ck.cocktail_pages_resize(S.pages, torch.tensor([-3, 0, 0, 0, 0], dtype=torch.int32).to(S.dev))   # three were refused
    for given in S.given:
        del given[0][-3:]
    S.fork([3, -1, 2, 3, 4])
    ck.cocktail_pages_compact(S.pages, S.pools())
    assert int(S.pages.refs[int((S.pages.refs > 0).sum()):].sum()) == 0
    S.step([1, 20, 1, 1, 1])
    # back out of the cache, into the mixed-precision one
    lens = [len(x) for x in S.given[0]]
    starts = torch.tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).to(S.dev)
    k, v = ck.cocktail_fp4_gather(S.caches[0], sum(lens), starts)
    assert np.array_equal(_f64(k), O.value(np.concatenate([np.stack([_f64(x[0]) for x in row]) for row in S.given[0]])))
    shape = ck.make_shape(1, 4, 2, d, 16, 32)
    plan = ck.cocktail_plan(shape, [lens[0]], np.full(lens[0] // 16, 16, np.uint8), ck.cocktail_default_workers(shape))
    mixed = ck.PackedCache(plan, S.dev)
    ck.cocktail_reorder_quantize(mixed, k[:lens[0]].transpose(0, 1)[None].contiguous(), v[:lens[0]].transpose(0, 1)[None].contiguous())
    q = torch.randn(1, 4, d, device=S.dev).half()
    a, _ = ck.cocktail_decode_attention(mixed, q)
    counts = [1, 0, 0, 0, 0]
    b, _ = ck.cocktail_fp4_attention(S.caches[0], q, torch.tensor([0, 1, 1, 1, 1, 1], dtype=torch.int32).to(S.dev))
    assert sum(counts) == 1 and (a.float() - b.float()).abs().max() <= 2e-3 * b.float().abs().max()


@gpu
def test_nothing_is_stored_without_room():
    S = Serving(2, 1, 128, 16, 4, torch.float16, layers=1)
    S.step([30, 20])
    before = S.caches[0].pool.clone()
    ck.cocktail_pages_resize(S.pages, torch.tensor([40, 1], dtype=torch.int32).to(S.dev), S.pools())
    x = torch.randn(41, 1, 128, device=S.dev).half()
    ck.cocktail_fp4_store(S.caches[0], x, x, torch.tensor([0, 40, 41], dtype=torch.int32).to(S.dev))
    assert torch.equal(S.caches[0].pool, before) and S.pages.seq_lens.tolist() == [30, 20]
    with pytest.raises(ck.CocktailError) as err:
        ck.cocktail_pages_check(S.pages)
    assert err.value.code == _lib.ESTATE
    S.step([1, 1])


@gpu
def test_a_generation_loop_in_a_captured_graph():
    """Room, store and attention of a step in a graph: every replay is a step, with eager work between them."""
    S = Serving(3, 2, 128, 16, 40, torch.float16, layers=1)
    S.step([20, 31, 16])
    one = torch.ones(3, dtype=torch.int32, device=S.dev)
    k, v, q = (torch.zeros(3, n, 128, device=S.dev, dtype=torch.float16) for n in (2, 2, 8))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ck.cocktail_pages_resize(S.pages, one, S.pools())
        ck.cocktail_fp4_store(S.caches[0], k, v)
        out, lse = ck.cocktail_fp4_attention(S.caches[0], q)
    with torch.cuda.graph(other, stream=side):               # a second graph over the same cache, with a workspace of its own
        out2, lse2 = ck.cocktail_fp4_attention(S.caches[0], q, sm_scale=0.01)
    torch.cuda.current_stream().wait_stream(side)
    for step in range(20):
        for t in (k, v, q):
            t.copy_(S.randn(*t.shape))
        graph.replay()
        for b in range(3):
            S.given[0][b].append((k[b].clone(), v[b].clone()))
        eager, eager_lse = ck.cocktail_fp4_attention(S.caches[0], q)
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse)
        S.verify(0, q, [1, 1, 1], out)
        other.replay()
        eager, _ = ck.cocktail_fp4_attention(S.caches[0], q, sm_scale=0.01)
        assert torch.equal(out2, eager)
    ck.cocktail_pages_check(S.pages)


@gpu
def test_calls_on_another_stream():
    B = Batch([500, 64], 2, 128, 16, torch.float16, seed=21)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q = B.query([1, 1], 4)
    s.wait_stream(torch.cuda.current_stream())
    ck.cocktail_fp4_store(B.cache, B.k, B.v, B.starts(B.lens), stream=s)
    out, lse = ck.cocktail_fp4_attention(B.cache, q, stream=s)
    k, v = ck.cocktail_fp4_gather(B.cache, 564, B.starts(B.lens), stream=s)
    ck.cocktail_pages_fork(B.pages, torch.tensor([0, 1], dtype=torch.int32).to(B.dev), stream=s)
    ck.cocktail_pages_check(B.pages, stream=s)
    B.check(q, [1, 1], out, lse)
    assert np.array_equal(_f64(k), O.value(_f64(B.k)))


@gpu
def test_calls_and_graphs_on_two_streams_at_once():
    """Two streams read one cache at the same time, eagerly and by graphs that are replayed side by side: nothing is shared but the cache."""
    B = Batch([5000, 3000, 700, 40], 4, 128, 16, torch.float16, seed=33)
    B.store_all()
    new = [4, 1, 3, 2]
    starts = B.starts(new)
    queries = [B.query(new, 8), B.query(new, 8)]
    call = lambda q: ck.cocktail_fp4_attention(B.cache, q, starts, max_new=4, max_len=5000)  # noqa: E731
    want = [call(q)[0].clone() for q in queries]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        got = []
        for s, q in zip(streams, queries):
            with torch.cuda.stream(s):
                got.append([call(q)[0] for _ in range(3)])
        torch.cuda.synchronize()
        assert all(torch.equal(x, want[i]) for i in range(2) for x in got[i])
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g, s, q in zip(graphs, streams, queries):
        with torch.cuda.graph(g, stream=s):
            outs.append(call(q)[0])
    for _ in range(10):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = call(queries[0])[0]
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0]) and all(torch.equal(o, w) for o, w in zip(outs, want))


@gpu
def test_most_sequences_with_most_rows():
    """4096 sequences, of which one needs four operands of queries of 128 channels: the most shared memory that a workgroup asks for."""
    lens, new = [5] * 4096, [0] * 4096
    lens[1234], new[1234], new[4000] = 700, 3, 1
    B = Batch(lens, 1, 128, 16, torch.float16, seed=34)
    B.store_all()
    q = B.query(new, 20)
    out, lse = ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=3)
    B.check(q, new, out, lse)


@gpu
def test_the_bindings_refusals():
    B = Batch([40, 20], 2, 128, 16, torch.float16)
    x = torch.zeros(4, 2, 128, device=B.dev, dtype=torch.float16)
    for bad in (x.float(), x.cpu(), x[:, :1], x[..., :64], x[..., ::2].repeat(1, 1, 2)[..., ::1][:, :, :64]):
        with pytest.raises(TypeError):
            ck.cocktail_fp4_store(B.cache, bad, x)
    for bad in (x.bfloat16(), x[:2], torch.zeros(4, 2, 256, device=B.dev, dtype=torch.float16)[..., :128]):
        with pytest.raises(ValueError):
            ck.cocktail_fp4_store(B.cache, x, bad)
    starts = torch.zeros(3, dtype=torch.int32, device=B.dev)
    for bad in (starts.long(), starts.cpu(), starts[:2]):
        with pytest.raises(TypeError):
            ck.cocktail_fp4_attention(B.cache, x, bad)
        with pytest.raises(TypeError):
            ck.cocktail_fp4_gather(B.cache, 4, bad)
    for bad in (torch.ones(2, device=B.dev), torch.ones(3, dtype=torch.int32, device=B.dev), torch.ones(2, dtype=torch.int32)):
        with pytest.raises(TypeError):
            ck.cocktail_pages_resize(B.pages, bad)
        with pytest.raises(TypeError):
            ck.cocktail_pages_fork(B.pages, bad)
    with pytest.raises(TypeError):
        ck.cocktail_pages_compact(B.pages, [B.cache.pool[1:]])
    with pytest.raises(ValueError):
        ck.cocktail_pages_compact(B.pages, [B.cache.pool, B.cache.pool.new_zeros(B.pages.num_pages, 16)])
    with pytest.raises(ValueError):
        ck.cocktail_fp4_attention(B.cache, x, out=x[:2])
    with pytest.raises(ValueError):
        ck.cocktail_fp4_attention(B.cache, x, lse=torch.zeros(4, 2, device=B.dev, dtype=torch.float16))
    with pytest.raises(TypeError):
        ck.Fp4Cache(B.pages, 2, 128, pool=torch.zeros(3, 3, device=B.dev, dtype=torch.uint8))
    with pytest.raises(ck.CocktailError):
        ck.Fp4Cache(B.pages, 2, 96)
    with pytest.raises(ck.CocktailError):
        ck.cocktail_fp4_attention(B.cache, torch.zeros(4, 3, 128, device=B.dev, dtype=torch.float16))
    # nothing to do
    empty = torch.zeros(0, 2, 128, device=B.dev, dtype=torch.float16)
    ck.cocktail_fp4_store(B.cache, empty, empty, starts)
    out, lse = ck.cocktail_fp4_attention(B.cache, empty, starts)
    assert out.shape == (0, 2, 128) and lse.shape == (0, 2)
