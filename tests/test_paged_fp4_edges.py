"""The paged 4-bit cache where it can go wrong besides what test_paged_fp4.py looks at: waits, threads, streams, far tails of a softmax, unusual queries,
starts and lengths."""
import contextlib
import ctypes as C
import re
import shutil
import subprocess
import threading
import time

import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck
from oracle import fp4_oracle as O
from paper_2503_23294_amd import _lib, paged
from test_device_code import _objdump
from test_paged_fp4 import DTYPES, Batch, _f64

gpu = pytest.mark.gpu


# ---- shared memory of the tile kernel ----------------------------------------------------------------------------------------


def test_first_products_of_a_tile_are_done_before_their_keys_are_replaced(tmp_path):
    """The logits of a workgroup's first 32 keys are products outside the loop, and the loop's first step puts other keys in their place: between
    the two the waves have to wait for each other."""
    tool = _objdump()
    lib = shutil.copy(_lib.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([tool, "--offloading", str(lib)], cwd=tmp_path, check=True, capture_output=True)
    kernels = 0
    for obj in sorted(tmp_path.glob("lib.so.*gfx950")):
        text = subprocess.run([tool, "-d", "--no-show-raw-insn", str(obj)], check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\w*fp4_tile_kernel\w*)>:\n(.*?)(?=^[0-9a-f]+ <\w+>:|\Z)", text, re.S | re.M):
            code = [line.split("//")[0].strip() for line in body.splitlines() if line.strip()]
            if not any(line.startswith("v_mfma") for line in code):
                continue
            kernels += 1
            steps = 8 if "ILi128E" in name else 4
            products = [i for i, line in enumerate(code) if line.startswith("v_mfma")][:steps]
            sums = {code[i].split()[1] for i in products}
            assert len(sums) == 1, f"{name}: the first {steps} products are not one chain: {sums}"
            behind = next(line for line in code[products[-1]:] if line.startswith(("s_barrier", "ds_write")))
            assert behind.startswith("s_barrier"), f"{name}: {behind} without a wait behind the first products"
    assert kernels == 4


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,kv_heads,rep", [([1100, 700], [514, 300], 4, 32),     # eight waves; 64 and 128 rows in the last tiles
                                                   ([300, 200, 90], [28, 33, 27], 2, 5),  # four waves; 12, 37 and 7 rows
                                                   ([700, 333], [683, 86], 4, 24)])       # four waves, keys not cut; 8 and 16 rows
def test_last_tiles_with_idle_waves(lens, new, kv_heads, rep, d):
    """Tiles of which at most half of the waves have rows; the same bits every time."""
    B = Batch(lens, kv_heads, d, 48, torch.float16, seed=d + rep, spread=2.0)
    B.store_all()
    q = B.query(new, rep)
    call = lambda: ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=max(new), max_len=max(lens))  # noqa: E731
    out, lse = call()
    B.check(q, new, out, lse)
    for _ in range(10):
        again, lse2 = call()
        assert torch.equal(out, again) and torch.equal(lse, lse2)


# ---- threads -------------------------------------------------------------------------------------------------------------------


class _SlowLib:
    """The library, but for the calls that launch several kernels: those take their time and note which workspace they have, and for how long."""

    def __init__(self):
        self.real, self.inside, self.mixed, self.calls = _lib.lib(), [], [], 0

    def __getattr__(self, name):
        if name not in ("cocktail_fp4_attention", "cocktail_pages_resize", "cocktail_pages_compact"):
            return getattr(self.real, name)
        place = {"cocktail_fp4_attention": 14, "cocktail_pages_resize": 5, "cocktail_pages_compact": 4}[name]

        def call(*args):
            me = (args[place], args[place] + args[place + 1])
            self.mixed += [(me, other) for other in self.inside if me[0] < other[1] and other[0] < me[1]]
            self.inside.append(me)
            self.calls += 1
            time.sleep(2e-4)
            self.inside.remove(me)
            return 0
        return call


def test_threads_do_not_share_a_workspace_at_the_same_time(monkeypatch):
    """Calls of several threads on one stream, of unlike sizes, so that the kept workspace is replaced by larger ones in between: no two calls
    are ever inside the library with memory in common, nor with memory that has been given up."""
    slow = _SlowLib()
    monkeypatch.setattr(paged, "lib", lambda: slow)
    monkeypatch.setattr(paged, "_here", lambda device, stream: 7)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    pages = ck.PageTable.of(i32(4, 2000), i32(4), i32(64), 16)
    cache = ck.Fp4Cache(pages, 2, 128)
    errors = []

    def work(seed):
        rng = np.random.default_rng(seed)
        try:
            for i in range(40):
                kind = rng.integers(0, 4)
                if kind == 0:
                    ck.cocktail_pages_resize(pages, i32(4))
                elif kind == 1:
                    ck.cocktail_pages_compact(pages)
                else:
                    n = int(rng.integers(1, 9))
                    ck.cocktail_fp4_attention(cache, torch.zeros(4 * n, 8, 128, dtype=torch.float16))
        except Exception as e:   # a thread's failure is the test's
            errors.append(e)
    threads = [threading.Thread(target=work, args=(seed,)) for seed in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert slow.calls == 160 and not slow.mixed


def test_the_caches_of_a_table_share_their_workspace(monkeypatch):
    """Layers attend one after the other on a stream: one workspace is enough for all of them, and for the calls on the table."""
    slow = _SlowLib()
    monkeypatch.setattr(paged, "lib", lambda: slow)
    monkeypatch.setattr(paged, "_here", lambda device, stream: 7)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    made, empty = [], torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: made.append(empty(*a, **k)) or made[-1])
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    pages = ck.PageTable.of(i32(4, 2000), i32(4), i32(64), 16)
    layers = [ck.Fp4Cache(pages, 2, 128) for _ in range(5)]
    q = torch.zeros(4, 8, 128, dtype=torch.float16)
    made.clear()
    for cache in layers:
        ck.cocktail_fp4_attention(cache, q)
    ck.cocktail_pages_resize(pages, i32(4))
    assert slow.calls == 6 and sum(x.dtype == torch.uint8 for x in made) == 1


@gpu
def test_two_threads_on_one_stream():
    """Two threads attend to one cache on the default stream, each with queries of its own: what they get is what one alone gets."""
    B = Batch([5000, 3000, 700, 40], 4, 128, 16, torch.float16, seed=51)
    B.store_all()
    new = [2, 1, 3, 1]
    starts = B.starts(new)
    queries = [B.query(new, 8) for _ in range(2)]
    call = lambda q: ck.cocktail_fp4_attention(B.cache, q, starts, max_new=3, max_len=5000)  # noqa: E731
    want = [[x.clone() for x in call(q)] for q in queries]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def work(i):
        try:
            got[i] = [call(queries[i]) for _ in range(300)]
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for i in range(2):
        assert len(got[i]) == 300
        assert all(torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1]) for out, lse in got[i])


# ---- streams -------------------------------------------------------------------------------------------------------------------


def test_what_is_used_on_another_stream_is_recorded_there(monkeypatch):
    """Every tensor that a call on a given stream works on, those of the table and the cache among them; none where no stream is given."""
    slow, seen = _SlowLib(), []
    quiet = type("Quiet", (), {"__getattr__": lambda self, name: (lambda *a: 0) if name in launches else getattr(slow, name)})()
    launches = ("cocktail_fp4_store", "cocktail_fp4_gather", "cocktail_pages_fork")
    monkeypatch.setattr(paged, "lib", lambda: quiet)
    monkeypatch.setattr(paged, "_here", lambda device, stream: None if stream is not None else 7)
    monkeypatch.setattr(paged, "_on", lambda device, stream: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: seen.append((self.data_ptr(), stream)), raising=False)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    f16 = lambda *shape: torch.zeros(shape, dtype=torch.float16)  # noqa: E731
    pages = ck.PageTable.of(i32(2, 5), i32(2), i32(8), 16)
    cache = ck.Fp4Cache(pages, 1, 64)
    table = [pages.table, pages.seq_lens, pages.refs, pages.status]
    k, v, q, out, lse, starts, delta = f16(4, 1, 64), f16(4, 1, 64), f16(4, 2, 64), f16(4, 2, 64), torch.zeros(4, 2), i32(3), i32(2)
    for call, used in ((lambda s: ck.cocktail_fp4_store(cache, k, v, starts, stream=s), [cache.pool, k, v, starts]),
                       (lambda s: ck.cocktail_fp4_gather(cache, 4, starts, out=(k, v), stream=s), [cache.pool, k, v, starts]),
                       (lambda s: ck.cocktail_fp4_gather(cache, 4, stream=s), [cache.pool]),
                       (lambda s: ck.cocktail_fp4_attention(cache, q, starts, out=out, lse=lse, stream=s), [cache.pool, q, starts, out, lse]),
                       (lambda s: ck.cocktail_fp4_attention(cache, q, stream=s), [cache.pool, q]),
                       (lambda s: ck.cocktail_pages_resize(pages, delta, stream=s), [delta]),
                       (lambda s: ck.cocktail_pages_fork(pages, delta, stream=s), [delta]),
                       (lambda s: ck.cocktail_pages_compact(pages, stream=s), [])):
        seen.clear()
        call(None)
        assert not seen
        call("a stream")
        assert {x for x, _ in seen} == {t.data_ptr() for t in table + used} and {s for _, s in seen} == {"a stream"}


@gpu
def test_tensors_that_are_dropped_behind_a_call_on_another_stream():
    """A stream that is busy gets calls whose arguments are temporaries of the current stream; these are dropped, and tensors of their sizes made and
    overwritten, before the calls take place."""
    lens, new = [500, 64, 130], [3, 1, 2]
    B = Batch(lens, 2, 128, 16, torch.bfloat16, seed=61)
    q = B.query(new, 4)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    B.store_all()
    want = [x.clone() for x in ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=3)]
    want += [x.clone() for x in ck.cocktail_fp4_gather(B.cache, sum(lens), B.starts(lens), dtype=B.dtype)]
    pool = B.cache.pool.clone()
    B.cache.pool.copy_(torch.from_numpy(B.junk))
    free = sum(r == 0 for r in B.pages.refs.tolist())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()

    def dropped(*shape_of):
        """Other tensors where the temporaries were."""
        return [torch.zeros_like(x) for x in shape_of for _ in range(4)]

    def there(*arrays):
        """Temporaries that the other stream waits for."""
        made = [(torch.from_numpy(a).to(B.dev) if isinstance(a, np.ndarray) else a.clone()) for a in arrays]
        s.wait_stream(torch.cuda.current_stream())
        return made
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    ck.cocktail_fp4_store(B.cache, *there(B.k, B.v, starts[0]), stream=s)
    keep = dropped(B.k, B.v, torch.from_numpy(starts[0]).to(B.dev))
    got = [*ck.cocktail_fp4_attention(B.cache, *there(q, starts[1]), max_new=3, stream=s)]
    keep += dropped(q, torch.from_numpy(starts[1]).to(B.dev))
    got += [*ck.cocktail_fp4_gather(B.cache, sum(lens), *there(starts[0]), dtype=B.dtype, stream=s)]
    keep += dropped(torch.from_numpy(starts[0]).to(B.dev))
    out, lse = torch.ones_like(q), torch.ones(sum(new), 8, device=B.dev)
    ck.cocktail_fp4_attention(B.cache, *there(q, starts[1]), max_new=3, out=out, lse=lse, stream=s)
    ck.cocktail_pages_fork(B.pages, *there(np.array([0, 1, 1], np.int32)), stream=s)
    ck.cocktail_pages_resize(B.pages, *there(np.array([0, 0, -64], np.int32)), [B.cache.pool], stream=s)
    keep += dropped(torch.zeros(3, dtype=torch.int32, device=B.dev))
    assert not s.query()       # still asleep: none of the calls has taken place
    ck.cocktail_pages_check(B.pages, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(B.cache.pool, pool)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert B.pages.seq_lens.tolist() == [500, 64, 0] and sum(r == 0 for r in B.pages.refs.tolist()) == free + 9
    assert len(keep) > 0


# ---- softmax -------------------------------------------------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("spread", [0.0, 0.3])
@pytest.mark.parametrize("tokens,new,max_len", [(131072, 1, 0), (131072, 1, 1), (131072, 6, 0), (131072, 10, 0), (131072, 16, 0), (32768, 40, 0)])
def test_the_tail_behind_one_large_key(tokens, new, max_len, spread):
    """One key with a logit that is 12 to 20 nats above those of all others (nearly alike), whose values are those that count: its own are zero, so
    that the result is the tail's share.  In one launch and two, with one to four operands of queries, and in tiles."""
    rep, d = 4, 64
    B = Batch([tokens], 1, d, 64, torch.float16, seed=new)
    gaps = (12.0, 15.0, 17.0, 17.5, 20.0)
    B.k.normal_(0, 1).mul_(0.14 / 0.3 * spread)
    B.v.normal_(0, 0.25).add_(1.0)
    B.k[0], B.v[0] = 1.0, 0.0
    B.store_all()
    k, v = ck.cocktail_fp4_gather(B.cache, tokens)
    k, v = k[:, 0].double(), v[:, 0].double()
    q = torch.empty(new, rep, d, device=B.dev, dtype=torch.float16)
    for i in range(new):
        for h in range(rep):
            q[i, h] = gaps[(i * rep + h) % 5] / d
    out, lse = ck.cocktail_fp4_attention(B.cache, q, max_len=max_len, sm_scale=1.0)
    s = q.double().view(-1, d) @ k.t()
    last = torch.arange(tokens - new, tokens, device=B.dev).repeat_interleave(rep)
    s.masked_fill_(torch.arange(tokens, device=B.dev)[None] > last[:, None], -float("inf"))
    total = torch.exp(s - s[:, :1]).sum(1, keepdim=True)
    w = torch.exp(s - s[:, :1]) / total
    want = w @ v
    # the result's rounding; the weights', in the sum over V and in the normaliser (2^-11 each); logits of up to 20, whose 64 products and sums in
    # binary32 are off by 68 * 2^-24 * 20 = 8.2e-5, and whose difference to the reference, 29 * 1.45 at most, by 2^-19; two sums of one term per 16 keys, in eight
    # parts at least where there are up to 64 rows; weights that are subnormals, results that are
    adds = tokens // 16 // (8 if new * rep <= 64 else 1) + 64
    bound = want.abs() * (3 * 2.0 ** -11 + 2 * (8.2e-5 + 2.0 ** -19) + 2 * adds * 2.0 ** -24) + tokens * 2.0 ** (-36 if new * rep <= 64 else -32) * v.abs().max() + 2.0 ** -25
    far = (out.double().view(-1, d) - want).abs()
    assert (far <= bound).all(), f"{(far / want.abs()).max()} of the result, {(far / bound).max()} of the bound"
    assert ((lse.double().view(-1) - torch.logsumexp(s, 1)).abs() <= 8.2e-5 + 2.0 ** -18 + adds * 2.0 ** -24).all()


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,rep,max_len", [([1, 30, 400], [1, 1, 1], 3, 400), ([30, 400, 90], [1, 1, 1], 3, 0), ([400, 33, 2], [2, 2, 2], 16, 0),
                                                  ([400, 390, 7] + [40 + 17 * i for i in range(20)], [3, 2, 3] + [3] * 20, 16, 0),
                                                  ([400, 64, 5] + [50 + 17 * i for i in range(20)], [4, 3, 4] + [4] * 20, 16, 0)])
def test_values_that_are_all_alike_come_out_as_they_are(lens, new, rep, max_len, d):
    """Up to 64 rows every weight goes into the normaliser as it goes into the sum over V, rounded: where a head's values are one vector for all keys the result
    is that vector, whatever the weights are.  Two sums of up to 400 terms in binary32, each off by 400 * 2^-23 = 4.8e-5 at most, are nearer to it
    than half the distance to the next fp16 below a power of two, 2^-13."""
    B = Batch(lens, 2, d, 16, torch.float16, seed=d + new[0])
    B.v[:] = torch.from_numpy(O.value(_f64(B.v[:1]))).to(B.dev, B.dtype)
    B.store_all()
    want = B.v[0].repeat_interleave(rep, 0)[None].expand(sum(new), -1, -1).clone()
    at = 0
    for t, n in zip(lens, new):
        want[at:at + max(0, n - t)] = 0
        at += n
    for scale in (1.0, 2.0, 4.0, 6.0, 8.0, 12.0):
        q = B.query(new, rep, scale)
        out, lse = ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=max(new), max_len=max_len)
        B.check(q, new, out, lse)
        assert torch.equal(out, want), scale


@gpu
@pytest.mark.parametrize("new", [1, 5, 40])
@pytest.mark.parametrize("power", [120, 125, 103, -105, -112, -120])
def test_bf16_queries_of_any_size(power, new):
    """Queries near the ends of bf16's range, and a scale that brings their logits back: results as for queries of ordinary size."""
    B = Batch([400, 77], 2, 128, 16, torch.bfloat16, seed=71)
    B.store_all()
    q = B.query([new, new], 4) * 2.0 ** power
    assert torch.isfinite(q).all()
    sm_scale = 2.0 ** -power / 128 ** 0.5
    out, lse = ck.cocktail_fp4_attention(B.cache, q, sm_scale=sm_scale)
    B.check(q, [new, new], out, lse, sm_scale)


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,new,rep", [([300, 120], [1, 1], 4), ([5000, 120], [3, 2], 16), ([5000, 120], [2, 4], 16), ([400, 399], [40, 70], 4),
                                          ([4000], [70], 4)])
def test_queries_that_are_not_finite(lens, new, rep, dtype):
    """A query with a NaN has a result and a logarithm of NaN, also where sums are held against limits; one with an infinity whose logits are none or infinite
    as well; all other queries have what they have without them.  Queries without keys have zeros, whatever they are."""
    B = Batch(lens, 2, 128, 16, DTYPES[dtype], seed=81)
    B.k[:, :, 7] = 1.5 * torch.sign(B.k[:, :, 7].float()).to(B.dtype) + 0.25       # channel 7 is stored as zero nowhere
    B.store_all()
    q = B.query(new, rep)
    call = lambda q: ck.cocktail_fp4_attention(B.cache, q, B.starts(new), max_new=max(new))  # noqa: E731
    out, lse = call(q)
    B.check(q, new, out, lse)
    heads, n = 2 * rep, sum(new)
    bad = [(0, 0), (0, heads - 1), (n - 1, 1), (n // 2, heads // 2)]
    for value in (float("nan"), float("inf"), -float("inf")):
        x = q.clone()
        for i, h in bad:
            x[i, h, 7] = value
        got, gl = call(x)
        same = torch.ones(n, heads, dtype=torch.bool, device=B.dev)
        for i, h in bad:
            same[i, h] = False
            assert torch.isnan(got[i, h]).all() and torch.isnan(gl[i, h]), (value, i, h)
        assert torch.equal(got[same], out[same]) and torch.equal(gl[same], lse[same])
    many = [t + 2 for t in lens] if max(lens) < 1000 else None
    if many:
        x = torch.full((sum(many), heads, 128), float("nan"), device=B.dev, dtype=B.dtype)
        got, gl = ck.cocktail_fp4_attention(B.cache, x, B.starts(many), max_new=max(many))
        at = 0
        for t, m in zip(lens, many):
            assert (got[at:at + 2] == 0).all() and torch.isneginf(gl[at:at + 2]).all()
            assert torch.isnan(got[at + 2:at + m]).all() and torch.isnan(gl[at + 2:at + m]).all()
            at += m


# ---- lengths and starts ----------------------------------------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("num_seqs", [2, 70])
@pytest.mark.parametrize("d,page,new", [(128, 16, [1, 1]), (64, 32, [10, 7]), (128, 16, [40, 3]), (64, 16, [9, 70])])
def test_lengths_beyond_the_table(d, page, new, num_seqs):
    """Lengths that the rows of the table cannot hold (they come from elsewhere: cocktail_pages_resize makes none): tokens behind the last column are
    not stored, read as zeros and are no keys; all others are what they are."""
    dev, room = torch.device("cuda:0"), 64
    rng = np.random.default_rng(d + num_seqs)
    for lens in ([70, 66], [64, 65], [2 ** 31 - 1, 100], [room + 2 * new[0] + 1, 2 ** 31 - 3]):
        columns = room // page
        table = rng.permutation(num_seqs * columns).astype(np.int32).reshape(num_seqs, columns)
        all_lens = np.zeros(num_seqs, np.int64)
        at = (0, num_seqs - 1)
        all_lens[list(at)] = lens
        counts = np.zeros(num_seqs, np.int64)
        counts[list(at)] = new
        t = lambda a: torch.from_numpy(a.astype(np.int32)).to(dev)  # noqa: E731
        pages = ck.PageTable.of(t(table), t(all_lens), t(np.ones(num_seqs * columns)), page)
        cache = ck.Fp4Cache(pages, 2, d)
        total = sum(new)
        starts = t(np.concatenate([[0], np.cumsum(counts)]))
        # what is there before: 64 tokens of every sequence
        k0, v0 = (torch.randn(num_seqs * room, 2, d, device=dev, dtype=torch.float16) for _ in range(2))
        pages.seq_lens.fill_(room)
        ck.cocktail_fp4_store(cache, k0, v0)
        want = [O.value(_f64(x)).reshape(num_seqs, room, 2, d) for x in (k0, v0)]
        pages.seq_lens.copy_(t(all_lens))
        k, v, q = (torch.randn(total, h, d, device=dev, dtype=torch.float16) for h in (2, 2, 4))
        ck.cocktail_fp4_store(cache, k, v, starts)
        gk, gv = ck.cocktail_fp4_gather(cache, total, starts)
        out, lse = ck.cocktail_fp4_attention(cache, q, starts, max_new=max(new))
        row = 0
        for b, length, n in zip(at, lens, new):
            read = np.zeros((2, n, 2, d))
            for i in range(n):
                pos = length - n + i
                if 0 <= pos < room:
                    for x, given in enumerate((k, v)):
                        want[x][b, pos] = read[x, i] = O.value(_f64(given[row + i]))
            rows = slice(row, row + n)
            assert np.array_equal(_f64(gk[rows]), read[0]) and np.array_equal(_f64(gv[rows]), read[1])
            # queries see at most what there is
            for i in range(n):
                seen = max(0, min(length - n + i + 1, room))
                w, wl, mean_v, _ = O.attention(_f64(q[row + i:row + i + 1]), want[0][b, :seen], want[1][b, :seen])
                # the result's rounding, the weights' twice; logits of unit normals add less than the slack of 2^-12
                assert (np.abs(_f64(out[row + i:row + i + 1]) - w) <= 2.0 ** -11 * np.abs(w) + 2.5 * 2.0 ** -11 * mean_v).all(), (b, i)
                if seen == 0:
                    assert torch.isneginf(lse[row + i]).all()
                else:
                    assert (np.abs(_f64(lse[row + i:row + i + 1]) - wl) <= 2.0 ** -12).all(), (b, i)
            row += n
        pages.seq_lens.fill_(room)
        gk, gv = ck.cocktail_fp4_gather(cache, num_seqs * room)
        assert np.array_equal(_f64(gk).reshape(want[0].shape), want[0]) and np.array_equal(_f64(gv).reshape(want[1].shape), want[1])


def test_tables_of_more_entries_than_32_bits_count_are_refused():
    """A resize adds up the pages that all sequences take; 2048 sequences of 2^20 pages are 2^31, whose sum would come out negative."""
    L = _lib.lib()
    n = C.c_size_t(0)
    for num_seqs, stride, page, code in ((2048, 1 << 20, 16, _lib.EINVAL), (4096, 1 << 20, 1, _lib.EINVAL), (2, 1 << 30, 1, _lib.EINVAL),
                                         (2047, 1 << 20, 16, 0), (4096, (1 << 19) - 1, 16, 0)):
        d = _lib.PageTableDesc(4096, 4096, 4096, 4096, num_seqs, stride, page, 64)
        assert L.cocktail_pages_workspace(C.byref(d), C.byref(n)) == code, (num_seqs, stride)
        if code:
            assert L.cocktail_pages_resize(C.byref(d), 4096, None, 0, 0, 4096, 1 << 20, None) == code
            assert b"2^31" in L.cocktail_last_error()


@gpu
@pytest.mark.parametrize("starts,valid", [([0, 40, 30, 30], [0]), ([0, 40, 65, 99], [0, 1]), ([-3, 40, 65, 98], [1, 2]), ([0, 40, 120, 98], [0]),
                                          ([5, 40, 65, 98], [0, 1, 2]), ([0, 40, -1, 98], [0]), ([0, 40, 65, 2 ** 31 - 1], [0, 1])])
@pytest.mark.parametrize("rep", [1, 4])
def test_ranges_that_are_none_next_to_good_ones(starts, valid, rep):
    """Sequences whose range is within the batch are stored, read back and attended to as ever; nothing is written for the others."""
    B = Batch([40, 30, 33], 2, 128, 16, torch.float16, seed=5)
    B.store_all()
    x, y = (torch.randn(98, 2, 128, device=B.dev).half() for _ in range(2))
    q = torch.randn(98, 2 * rep, 128, device=B.dev).half()
    dev_starts = torch.tensor(starts, dtype=torch.int32, device=B.dev)
    ck.cocktail_fp4_store(B.cache, x, y, dev_starts)
    gk, gv = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    ck.cocktail_fp4_gather(B.cache, 98, dev_starts, out=(gk, gv))
    out, lse = torch.full_like(q, 7.0), torch.full((98, 2 * rep), 7.0, device=B.dev)
    ck.cocktail_fp4_attention(B.cache, q, dev_starts, out=out, lse=lse)
    others = torch.ones(98, dtype=torch.bool)
    for b in valid:
        n = starts[b + 1] - starts[b]
        rows = slice(starts[b], starts[b + 1])
        others[rows] = False
        mine = B.rows(b)
        last = slice(mine.stop - n, mine.stop)
        B.k[last], B.v[last] = x[rows], y[rows]
        assert np.array_equal(_f64(gk[rows]), O.value(_f64(x[rows]))) and np.array_equal(_f64(gv[rows]), O.value(_f64(y[rows])))
        B.check(q[rows], [n if i == b else 0 for i in range(3)], out[rows], lse[rows])
    for t in (gk, gv, out, lse):
        assert (t.cpu()[others] == 7.0).all()
    # the pool: what has been stored, and nothing else
    k, v = ck.cocktail_fp4_gather(B.cache, 103, B.starts(B.lens))
    assert np.array_equal(_f64(k), O.value(_f64(B.k))) and np.array_equal(_f64(v), O.value(_f64(B.v)))


@gpu
def test_workspaces_that_grow_while_graphs_live():
    """Eager calls of unlike sizes on one stream, each larger one with a new workspace, between replays of graphs that were captured when the
    workspaces were smaller; resizes and compactions use the same ones."""
    B = Batch([3000, 900, 40], 2, 128, 16, torch.float16, seed=91)
    B.store_all()
    sizes = [[1, 1, 1], [4, 1, 2], [8, 8, 8], [70, 3, 20], [16, 16, 16]]
    queries = [B.query(new, 4) for new in sizes]
    call = lambda i: ck.cocktail_fp4_attention(B.cache, queries[i], B_starts[i], max_new=max(sizes[i]), max_len=3000)  # noqa: E731
    B_starts = [B.starts(new) for new in sizes]
    want, graphs, outs = [], [], []
    side = torch.cuda.Stream()
    for i in range(len(sizes)):
        out, lse = call(i)
        B.check(queries[i], sizes[i], out, lse)
        want.append((out.clone(), lse.clone()))
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            outs.append(call(i))
        graphs.append(graph)
    nothing = torch.zeros(3, dtype=torch.int32, device=B.dev)
    for turn in range(6):
        for i in (turn % 5, (turn + 2) % 5, 4 - turn % 5):
            outs[i][0].zero_()
            outs[i][1].zero_()
            graphs[i].replay()
            got = call((i + turn) % 5)
            ck.cocktail_pages_resize(B.pages, nothing, [B.cache.pool])
            assert torch.equal(got[0], want[(i + turn) % 5][0]) and torch.equal(got[1], want[(i + turn) % 5][1])
            assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])
        ck.cocktail_pages_compact(B.pages, [B.cache.pool])


@gpu
def test_calls_on_a_given_stream_while_it_is_captured():
    """stream= names the stream that is captured, or one that joins the capture: tensors are recorded there as outside of a capture, and replays give what
    eager calls give, also after temporaries of the capture have been dropped."""
    B = Batch([2500, 64, 130], 2, 64, 16, torch.float16, seed=101)
    B.store_all()
    new = [2, 1, 1]
    q, starts = B.query(new, 6), B.starts(new)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        first = ck.cocktail_fp4_attention(B.cache, q * 1.0, starts, max_new=2, stream=side)
        other.wait_stream(side)
        second = ck.cocktail_fp4_attention(B.cache, q, starts, max_new=2, sm_scale=0.01, stream=other)
        side.wait_stream(other)
    for _ in range(5):
        q.copy_(B.query(new, 6))
        graph.replay()
        for got, scale in ((first, 0.0), (second, 0.01)):
            out, lse = ck.cocktail_fp4_attention(B.cache, q, starts, max_new=2, sm_scale=scale)
            assert torch.equal(got[0], out) and torch.equal(got[1], lse)
        junk = [torch.randn_like(q) for _ in range(8)]
        torch.cuda.synchronize()
        del junk
