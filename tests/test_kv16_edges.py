"""The paged 16-bit cache and beam search where they can go wrong besides what test_kv16.py and test_beam.py look at: lengths and ranges, large pools,
streams, threads, graphs, far tails of a softmax; and runs of the operators together, as they are used."""
import contextlib
import ctypes as C
import math
import threading

import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck
from oracle import cocktail_oracle as CO
from oracle import fp4_oracle as F
from oracle import kv16_oracle as O
from paper_2503_23294_amd import _lib, beam, kv16, paged
from test_kv16 import DTYPES, Batch, _check_turned, _f64, _freq, _rotation

gpu = pytest.mark.gpu


# ---- threads and streams, without a GPU --------------------------------------------------------------------------------------------


class _QuietLib:
    """The library, but for the calls that launch kernels: those do nothing, and note the workspaces that attention works in."""

    def __init__(self):
        self.real, self.inside, self.mixed, self.calls = _lib.lib(), [], [], 0

    def __getattr__(self, name):
        if name == "cocktail_kv16_attention":
            def call(*args):
                me = (args[12], args[12] + args[13])
                self.mixed += [(me, other) for other in self.inside if me[0] < other[1] and other[0] < me[1]]
                self.inside.append(me)
                self.calls += 1
                threading.Event().wait(2e-4)
                self.inside.remove(me)
                return 0
            return call
        if name in ("cocktail_kv16_append", "cocktail_beam_select", "cocktail_beam_reorder", "cocktail_pages_resize"):
            return lambda *args: 0
        return getattr(self.real, name)


@pytest.fixture
def quiet(monkeypatch):
    lib = _QuietLib()
    for module in (kv16, beam, paged):
        monkeypatch.setattr(module, "lib", lambda: lib)
        monkeypatch.setattr(module, "_here", lambda device, stream: None if stream is not None else 7)
        monkeypatch.setattr(module, "_on", lambda device, stream: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: None, raising=False)      # what the index of a CPU device is
    return lib


def test_threads_do_not_share_a_workspace_at_the_same_time(quiet):
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    pages = ck.PageTable.of(i32(4, 2000), i32(4), i32(64), 16)
    caches = [ck.Kv16Cache(pages, 2, 128) for _ in range(2)]
    errors = []

    def work(seed):
        rng = np.random.default_rng(seed)
        try:
            for _ in range(40):
                ck.cocktail_kv16_attention(caches[int(rng.integers(0, 2))], torch.zeros(4 * int(rng.integers(1, 9)), 8, 128, dtype=torch.float16))
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=work, args=(seed,)) for seed in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert quiet.calls == 160 and not quiet.mixed


def test_what_is_used_on_another_stream_is_recorded_there(quiet, monkeypatch):
    seen = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: seen.append((self.data_ptr(), stream)), raising=False)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    f16 = lambda *shape: torch.zeros(shape, dtype=torch.float16)  # noqa: E731
    pages = ck.PageTable.of(i32(2, 5), i32(2), i32(8), 16)
    cache = ck.Kv16Cache(pages, 1, 64)
    pools = [pages.table, pages.seq_lens, pages.refs, pages.status, cache.k, cache.v]
    k, v, q, q_out, out, lse, starts, positions = f16(4, 1, 64), f16(4, 1, 64), f16(4, 2, 64), f16(4, 2, 64), f16(4, 2, 64), torch.zeros(4, 2), i32(3), i32(4)
    rot = ck.Rotation(torch.zeros(32, dtype=torch.float64))
    logits, scores, ended = torch.zeros(4, 9), torch.zeros(4), torch.zeros(4, dtype=torch.bool)
    chosen = i32(2, 2), i32(2, 2), torch.zeros(2, 2), torch.zeros(2, 2, dtype=torch.bool)
    source, a, b, c = i32(4), f16(4, 8), f16(4, 8), f16(4, 3)
    for call, used in ((lambda s: ck.cocktail_kv16_append(cache, k, v, starts, stream=s), pools + [k, v, starts]),
                       (lambda s: ck.cocktail_kv16_append(cache, k, v, starts, rot, q=q, positions=positions, q_out=q_out, stream=s),
                        pools + [k, v, starts, rot.inv_freq, q, positions, q_out]),
                       (lambda s: ck.cocktail_kv16_attention(cache, q, starts, out=out, lse=lse, stream=s), pools + [q, starts, out, lse]),
                       (lambda s: ck.cocktail_kv16_attention(cache, q, stream=s), pools + [q]),
                       (lambda s: ck.cocktail_beam_select(logits, scores, 2, eos=1, finished=ended, out=chosen, stream=s), [logits, scores, ended, *chosen]),
                       (lambda s: ck.cocktail_beam_reorder(source, [a, c], stream=s), [source, a, c]),
                       (lambda s: ck.cocktail_beam_reorder(source, [a], out=[b], stream=s), [source, a, b])):
        seen.clear()
        call(None)
        assert not seen
        call("a stream")
        assert {x for x, _ in seen} == {t.data_ptr() for t in used} and {s for _, s in seen} == {"a stream"}


def test_states_that_overlap_are_refused(quiet):
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    x = torch.zeros(8, 6)
    source = i32(4)
    for states, out in (([x[:4], x[3:7]], None), ([x[:4], x[:4]], None), ([x[:4]], [x[2:6]]), ([x[:4], x[4:]], [torch.zeros(4, 6), x[3:7]]),
                        ([x[:4], x[:4]], [x[4:], x[4:]])):
        with pytest.raises(ValueError):
            ck.cocktail_beam_reorder(source, states, out=out)
    ck.cocktail_beam_reorder(source, [x[:4], x[4:]])
    ck.cocktail_beam_reorder(source, [x[:4], x[:4]], out=[x[4:], torch.zeros(4, 6)])       # read twice
    for states, out in (([x[:3]], None), ([x[:4, :3]], None), ([x[:4]], [])):
        with pytest.raises((TypeError, ValueError)):
            ck.cocktail_beam_reorder(source, states, out=out)
    with pytest.raises(ValueError):
        ck.cocktail_beam_reorder(source, [x[:4]], out=[x[4:].int()])
    with pytest.raises(TypeError):
        ck.cocktail_beam_reorder(source.long(), [x[:4]])


# ---- lengths, ranges, pools ------------------------------------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("num_seqs", [2, 70])
@pytest.mark.parametrize("d,page,new", [(128, 16, [1, 1]), (64, 32, [10, 7]), (128, 16, [40, 3]), (64, 16, [9, 70])])
def test_lengths_beyond_the_table(d, page, new, num_seqs):
    """Lengths that the rows of the table cannot hold: tokens behind the last column are not stored and are no keys; the rest is what it is."""
    dev, room = torch.device("cuda:0"), 64
    rng = np.random.default_rng(d + num_seqs)
    for lens in ([70, 66], [64, 65], [2 ** 31 - 1, 100], [room + 2 * new[0] + 1, 2 ** 31 - 3]):
        columns = room // page
        table = rng.permutation(num_seqs * columns).astype(np.int32).reshape(num_seqs, columns)
        all_lens, counts = np.zeros(num_seqs, np.int64), np.zeros(num_seqs, np.int64)
        at = (0, num_seqs - 1)
        all_lens[list(at)], counts[list(at)] = lens, new
        t = lambda a: torch.from_numpy(a.astype(np.int32)).to(dev)  # noqa: E731
        pages = ck.PageTable.of(t(table), t(all_lens), t(np.ones(num_seqs * columns)), page)
        cache = ck.Kv16Cache(pages, 2, d)
        total = sum(new)
        starts = t(np.concatenate([[0], np.cumsum(counts)]))
        k0, v0 = (torch.randn(num_seqs * room, 2, d, device=dev, dtype=torch.float16) for _ in range(2))
        pages.seq_lens.fill_(room)
        ck.cocktail_kv16_append(cache, k0, v0)
        want = [_f64(x).reshape(num_seqs, room, 2, d) for x in (k0, v0)]
        pages.seq_lens.copy_(t(all_lens))
        k, v, q = (torch.randn(total, h, d, device=dev, dtype=torch.float16) for h in (2, 2, 4))
        ck.cocktail_kv16_append(cache, k, v, starts)
        out, lse = ck.cocktail_kv16_attention(cache, q, starts, max_new=max(new))
        row = 0
        for b, length, n in zip(at, lens, new):
            for i in range(n):
                pos = length - n + i
                if 0 <= pos < room:
                    want[0][b, pos], want[1][b, pos] = _f64(k[row + i]), _f64(v[row + i])
            for i in range(n):
                seen = max(0, min(length - n + i + 1, room))
                w, wl, mean_v, _ = F.attention(_f64(q[row + i:row + i + 1]), want[0][b, :seen], want[1][b, :seen])
                # the result's rounding, the weights' twice; logits of unit normals add less than the slack of 2^-12
                assert (np.abs(_f64(out[row + i:row + i + 1]) - w) <= 2.0 ** -11 * np.abs(w) + 2.5 * 2.0 ** -11 * mean_v).all(), (b, i)
                if seen == 0:
                    assert torch.isneginf(lse[row + i]).all()
                else:
                    assert (np.abs(_f64(lse[row + i:row + i + 1]) - wl) <= 2.0 ** -12).all(), (b, i)
            row += n
        ids = torch.from_numpy(table.astype(np.int64)).to(dev)
        for pool, w in zip(cache.pools, want):
            assert np.array_equal(_f64(pool[ids].transpose(2, 3).flatten(1, 2)), w)


@gpu
@pytest.mark.parametrize("starts,valid", [([0, 40, 30, 30], [0]), ([0, 40, 65, 99], [0, 1]), ([-3, 40, 65, 98], [1, 2]), ([0, 40, 120, 98], [0]),
                                          ([5, 40, 65, 98], [0, 1, 2]), ([0, 40, -1, 98], [0]), ([0, 40, 65, 2 ** 31 - 1], [0, 1])])
@pytest.mark.parametrize("rep", [1, 4])
def test_ranges_that_are_none_next_to_good_ones(starts, valid, rep):
    """Sequences whose range is within the batch are stored and attended to as ever; nothing is written for the others."""
    B = Batch([40, 30, 33], 2, 128, 16, torch.float16, seed=5)
    B.store_all()
    x, y = (torch.randn(98, 2, 128, device=B.dev).half() for _ in range(2))
    q = torch.randn(98, 2 * rep, 128, device=B.dev).half()
    dev_starts = torch.tensor(starts, dtype=torch.int32, device=B.dev)
    turned = torch.full_like(q, 7.0)
    still = ck.Rotation(torch.zeros(8, dtype=torch.float64, device=B.dev))       # turns nothing
    before = [p.clone() for p in B.cache.pools]
    ck.cocktail_kv16_append(B.cache, x, y, dev_starts, still, q=q, q_out=turned)
    out, lse = torch.full_like(q, 7.0), torch.full((98, 2 * rep), 7.0, device=B.dev)
    ck.cocktail_kv16_attention(B.cache, q, dev_starts, out=out, lse=lse)
    others = torch.ones(98, dtype=torch.bool)
    for b in valid:
        n = starts[b + 1] - starts[b]
        rows = slice(starts[b], starts[b + 1])
        others[rows] = False
        mine = B.rows(b)
        last = slice(mine.stop - n, mine.stop)
        B.k[last], B.v[last] = x[rows], y[rows]
        assert torch.equal(turned[rows], q[rows])
        B.check(q[rows], [n if i == b else 0 for i in range(3)], out[rows], lse[rows])
    for t in (turned, out, lse):
        assert (t.cpu()[others] == 7.0).all()
    for pool, old, rows in zip(B.cache.pools, before, (B.k, B.v)):
        for b in range(3):
            for pos in range(B.lens[b]):
                old[int(B.table[b, pos // 16]), :, pos % 16] = rows[B.rows(b)][pos]
        assert torch.equal(pool.view(torch.int16), old.view(torch.int16))


@gpu
@pytest.mark.parametrize("num_seqs", [70, 1500, 4096])
def test_few_active_sequences_in_a_large_table(num_seqs):
    rng = np.random.default_rng(num_seqs)
    active = np.sort(rng.choice(num_seqs, 6, replace=False))
    lens, new = np.zeros(num_seqs, int), np.zeros(num_seqs, int)
    lens[active], new[active] = [300, 0, 77, 1000, 16, 130], [1, 1, 2, 1, 1, 1]
    for most in (2, 60):
        new[active[-1]] = most - 1
        B = Batch(lens.tolist(), 2, 64, 16, torch.bfloat16, seed=num_seqs)
        B.store_all()
        q = B.query(new.tolist(), 4)
        for max_len in (1000, 0):
            out, lse = ck.cocktail_kv16_attention(B.cache, q, B.starts(new.tolist()), max_new=most, max_len=max_len)
            B.check(q, new.tolist(), out, lse)


@gpu
def test_most_sequences_with_most_rows():
    lens, new = [5] * 4096, [0] * 4096
    lens[1234], new[1234], new[4000] = 700, 3, 1
    B = Batch(lens, 1, 128, 16, torch.float16, seed=34)
    B.store_all()
    q = B.query(new, 20)
    out, lse = ck.cocktail_kv16_attention(B.cache, q, B.starts(new), max_new=3)
    B.check(q, new, out, lse)


@gpu
def test_pools_beyond_32_bits():
    """Pages whose bytes lie beyond 2^32, in pools of 4.3 GB each."""
    dev = torch.device("cuda:0")
    num_pages, page, h, d = 16500, 64, 16, 128
    last = num_pages - 1
    table = torch.tensor([[last, last - 7, 3, -1], [last - 100, 9, last - 1, 8]], dtype=torch.int32, device=dev)
    lens = [130, 250]
    refs = torch.zeros(num_pages, dtype=torch.int32, device=dev)
    refs[table[table >= 0].long()] = 1
    pages = ck.PageTable.of(table, torch.tensor(lens, dtype=torch.int32, device=dev), refs, page)
    cache = ck.Kv16Cache(pages, h, d, torch.bfloat16)
    assert cache.k.nbytes > 1 << 32
    k, v, q = (torch.randn(380, n, d, device=dev, dtype=torch.bfloat16) for n in (h, h, 2 * h))
    starts = torch.tensor([0, 130, 380], dtype=torch.int32, device=dev)
    ck.cocktail_kv16_append(cache, k, v, starts)
    for b, at in ((0, 0), (1, 130)):
        pos = torch.arange(lens[b], device=dev)
        rows = cache.v[table[b, pos // page].long(), :, pos % page]
        assert torch.equal(rows, v[at:at + lens[b]])
    for new in ([1, 1], [130, 250]):
        qs = torch.cat([q[130 - new[0]:130], q[380 - new[1]:]])
        out, lse = ck.cocktail_kv16_attention(cache, qs, torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device=dev), max_new=max(new))
        row = 0
        for (at, t), n in zip(((0, 130), (130, 250)), new):
            w, wl, mean_v, _ = F.attention(_f64(qs[row:row + n]), _f64(k[at:at + t]), _f64(v[at:at + t]))
            # the result's rounding and the weights' twice, and logits of unit normals as above
            assert (np.abs(_f64(out[row:row + n]) - w) <= 2.0 ** -8 * np.abs(w) + 2.1 * 2.0 ** -8 * mean_v).all()
            assert (np.abs(_f64(lse[row:row + n]) - wl) <= 2.0 ** -12).all()
            row += n


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
    k, v = B.k[:, 0].double(), B.v[:, 0].double()
    q = torch.empty(new, rep, d, device=B.dev, dtype=torch.float16)
    for i in range(new):
        for h in range(rep):
            q[i, h] = gaps[(i * rep + h) % 5] / d
    out, lse = ck.cocktail_kv16_attention(B.cache, q, max_len=max_len, sm_scale=1.0)
    s = q.double().view(-1, d) @ k.t()
    last = torch.arange(tokens - new, tokens, device=B.dev).repeat_interleave(rep)
    s.masked_fill_(torch.arange(tokens, device=B.dev)[None] > last[:, None], -float("inf"))
    w = torch.softmax(s, dim=1)
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
@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "fp16"), (128, "bf16")])
@pytest.mark.parametrize("lens,new,rep,max_len", [([1, 30, 400], [1, 1, 1], 3, 400), ([30, 400, 90], [1, 1, 1], 3, 0), ([400, 33, 2], [2, 2, 2], 16, 0),
                                                  ([400, 64, 5] + [50 + 17 * i for i in range(20)], [4, 3, 4] + [4] * 20, 16, 0)])
def test_values_that_are_all_alike_come_out_as_they_are(lens, new, rep, max_len, d, dtype):
    """Up to 64 rows every weight goes into the normaliser as it goes into the sum over V, rounded: where a head's values are one vector for all keys the result
    is that vector, whatever the weights are.  Two sums of up to 400 terms in binary32, each off by 400 * 2^-23 = 4.8e-5 at most, are nearer to it
    than half the distance to the next fp16 below a power of two, 2^-13."""
    B = Batch(lens, 2, d, 16, DTYPES[dtype], seed=d + new[0])
    B.v[:] = B.v[:1]
    B.store_all()
    want = B.v[0].repeat_interleave(rep, 0)[None].expand(sum(new), -1, -1).clone()
    at = 0
    for t, n in zip(lens, new):
        want[at:at + max(0, n - t)] = 0
        at += n
    for scale in (1.0, 4.0, 12.0):
        q = B.query(new, rep, scale)
        out, lse = ck.cocktail_kv16_attention(B.cache, q, B.starts(new), max_new=max(new), max_len=max_len)
        B.check(q, new, out, lse)
        assert torch.equal(out, want), scale


# ---- streams, threads and graphs -----------------------------------------------------------------------------------------------------


@gpu
def test_a_step_in_a_captured_graph():
    """Room, rotated append, attention and, beside them, a step of a search in graphs: every replay is a step, with eager work between them."""
    dev = torch.device("cuda:0")
    pages = ck.PageTable(3, 400, 80, 16, dev)
    cache = ck.Kv16Cache(pages, 2, 128, torch.bfloat16)
    rot = _rotation(128)
    given = [([], []) for _ in range(3)]

    def keep(k, v, counts, firsts):
        at = 0
        for b, n in enumerate(counts):
            given[b][0].append(O.rotate(_f64(k[at:at + n]), np.arange(firsts[b], firsts[b] + n), _freq(128), False))
            given[b][1].append(_f64(v[at:at + n]))
            at += n
    lens = [20, 31, 16]
    k, v, q = (torch.randn(67, n, 128, device=dev, dtype=torch.bfloat16) for n in (2, 2, 8))
    ck.cocktail_pages_resize(pages, torch.tensor(lens, dtype=torch.int32, device=dev), cache.pools)
    ck.cocktail_kv16_append(cache, k, v, torch.tensor([0, 20, 51, 67], dtype=torch.int32, device=dev), rot)
    keep(k, v, lens, [0, 0, 0])
    one = torch.ones(3, dtype=torch.int32, device=dev)
    k, v, q = (torch.zeros(3, n, 128, device=dev, dtype=torch.bfloat16) for n in (2, 2, 8))
    logits, scores = torch.zeros(6, 5000, device=dev), torch.zeros(6, device=dev)
    state = torch.zeros(6, 700, device=dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ck.cocktail_pages_resize(pages, one, cache.pools)
        turned = ck.cocktail_kv16_append(cache, k, v, rotation=rot, q=q)
        out, lse = ck.cocktail_kv16_attention(cache, turned)
    with torch.cuda.graph(other, stream=side):
        chosen = ck.cocktail_beam_select(logits, scores, 2)
        ck.cocktail_beam_reorder(chosen[0], [state])
    torch.cuda.current_stream().wait_stream(side)
    for step in range(12):
        for t in (k, v, q, logits, scores, state):
            t.copy_(torch.randn_like(t))
        before = state.clone()
        graph.replay()
        other.replay()
        keep(k, v, [1, 1, 1], lens)
        want = ck.cocktail_beam_select(logits, scores, 2)
        assert all(torch.equal(a, b) for a, b in zip(chosen, want))
        assert torch.equal(state, before[want[0].view(-1).long()])
        _check_turned(turned, q, lens, _freq(128), False, 1.0, torch.bfloat16)
        eager, eager_lse = ck.cocktail_kv16_attention(cache, turned)
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse)
        lens = [n + 1 for n in lens]
        for b in range(3):
            w, _, mean_v, size = F.attention(_f64(turned[b:b + 1]), np.concatenate(given[b][0]), np.concatenate(given[b][1]))
            # K was rounded once more than the oracle's: half a step in every product
            far = np.abs(_f64(out[b:b + 1]) - w)
            assert (far <= 2.0 ** -8 * np.abs(w) + 2 * (2.0 ** -8 + 2.0 ** -8 * size[..., None] + 2.0 ** -12) * mean_v).all()
    ck.cocktail_pages_check(pages)
    assert pages.seq_lens.tolist() == lens


@gpu
def test_calls_and_graphs_on_two_streams_at_once():
    B = Batch([5000, 3000, 700, 40], 4, 128, 16, torch.bfloat16, seed=33)
    B.store_all()
    new = [4, 1, 3, 2]
    starts = B.starts(new)
    queries = [B.query(new, 8), B.query(new, 8)]
    rows = [torch.randn(12, 30011, device=B.dev) for _ in range(2)]
    scores = torch.zeros(12, device=B.dev)
    call = lambda i: [*ck.cocktail_kv16_attention(B.cache, queries[i], starts, max_new=4, max_len=5000), *ck.cocktail_beam_select(rows[i], scores, 4)]  # noqa: E731
    want = [[x.clone() for x in call(i)] for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        got = []
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append([call(i) for _ in range(3)])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for i in range(2) for result in got[i] for x, y in zip(result, want[i]))
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for i, (g, s) in enumerate(zip(graphs, streams)):
        with torch.cuda.graph(g, stream=s):
            outs.append(call(i))
    for _ in range(10):
        for result in outs:
            for o in result:
                o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = call(0)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(eager, want[0]))
        assert all(torch.equal(x, y) for result, w in zip(outs, want) for x, y in zip(result, w))


@gpu
def test_tensors_that_are_dropped_behind_a_call_on_another_stream():
    """A stream that is busy gets calls whose arguments are temporaries of the current stream; these are dropped, and tensors of their sizes made and
    overwritten, before the calls take place."""
    lens, new = [500, 64, 130], [3, 1, 2]
    B = Batch(lens, 2, 128, 16, torch.bfloat16, seed=61)
    q, rot = B.query(new, 4), _rotation(128)
    starts = [np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (lens, new)]
    rows, scores, state = torch.randn(6, 9000, device=B.dev), torch.randn(6, device=B.dev), torch.randn(6, 4000, device=B.dev)
    all_q = B.query(lens, 4)
    want = [ck.cocktail_kv16_append(B.cache, B.k, B.v, B.starts(lens), rot, q=all_q)]
    want += [*ck.cocktail_kv16_attention(B.cache, q, B.starts(new), max_new=3)]
    want += [*ck.cocktail_beam_select(rows, scores, 3)]
    want += ck.cocktail_beam_reorder(want[3].view(-1), [state], out=[torch.empty_like(state)])
    pools = [p.clone() for p in B.cache.pools]
    for p in B.cache.pools:
        p.zero_()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()

    def there(*arrays):
        made = [(torch.from_numpy(a).to(B.dev) if isinstance(a, np.ndarray) else a.clone()) for a in arrays]
        s.wait_stream(torch.cuda.current_stream())
        return made

    def dropped(*shape_of):
        return [torch.zeros_like(x) for x in shape_of for _ in range(4)]
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)

    def append(k, v, first, q_all, freq):
        return ck.cocktail_kv16_append(B.cache, k, v, first, ck.Rotation(freq), q=q_all, stream=s)
    got = [append(*there(B.k, B.v, starts[0], all_q, rot.inv_freq))]
    junk = dropped(B.k, B.v, all_q, rot.inv_freq, torch.from_numpy(starts[0]).to(B.dev))
    got += [*ck.cocktail_kv16_attention(B.cache, *there(q, starts[1]), max_new=3, stream=s)]
    junk += dropped(q, torch.from_numpy(starts[1]).to(B.dev))
    got += [*ck.cocktail_beam_select(*there(rows, scores), 3, stream=s)]
    junk += dropped(rows, scores)
    got += ck.cocktail_beam_reorder(got[3].view(-1), there(state), out=[torch.empty_like(state)], stream=s)
    junk += dropped(state)
    assert not s.query()       # still asleep: none of the calls has taken place
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and len(junk) > 0
    for pool, old in zip(B.cache.pools, pools):
        for b in range(3):
            assert torch.equal(B.pool_rows(b, 0, lens[b], pool), B.pool_rows(b, 0, lens[b], old))


@gpu
def test_two_threads_on_one_stream():
    B = Batch([5000, 3000, 700, 40], 4, 128, 16, torch.float16, seed=51)
    B.store_all()
    new = [2, 1, 3, 1]
    starts = B.starts(new)
    queries = [B.query(new, 8) for _ in range(2)]
    rows = [torch.randn(12, 30011, device=B.dev) for _ in range(2)]
    scores = torch.zeros(12, device=B.dev)
    call = lambda i: [*ck.cocktail_kv16_attention(B.cache, queries[i], starts, max_new=3, max_len=5000), *ck.cocktail_beam_select(rows[i], scores, 4)]  # noqa: E731
    want = [[x.clone() for x in call(i)] for i in range(2)]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def work(i):
        try:
            got[i] = [call(i) for _ in range(200)]
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert all(len(g) == 200 for g in got)
    assert all(torch.equal(x, y) for i in range(2) for result in got[i] for x, y in zip(result, want[i]))


# ---- together ------------------------------------------------------------------------------------------------------------------


@gpu
def test_a_prefill_in_chunks_that_is_quantized_then():
    """Prompts come in chunks: room, rotated append, attention over what is there; then the pages are reordered and quantized, and a decode step over the packed
    cache agrees with the oracle's on the same keys and values, as it agrees with attention over the pages where all chunks stay in fp16."""
    dev = torch.device("cuda:0")
    lens, hq, hkv, d, chunk = [353, 256], 8, 2, 128, 32
    rng = np.random.default_rng(4)
    pages = ck.PageTable(2, 400, 60, 16, dev)
    cache = ck.Kv16Cache(pages, hkv, d)
    rot = _rotation(d)
    make = lambda h: [torch.from_numpy(rng.standard_normal((n, h, d))).to(dev, torch.float16) for n in lens]  # noqa: E731
    k, v, q = make(hkv), make(hkv), make(hq)
    done = [0, 0]
    for piece in ([100, 200], [200, 0], [53, 56]):
        part = lambda x: torch.cat([x[b][done[b]:done[b] + n] for b, n in enumerate(piece)])  # noqa: E731
        starts = torch.tensor([0, piece[0], sum(piece)], dtype=torch.int32, device=dev)
        ck.cocktail_pages_resize(pages, torch.tensor(piece, dtype=torch.int32, device=dev), cache.pools)
        turned = ck.cocktail_kv16_append(cache, part(k), part(v), starts, rot, q=part(q))
        out, lse = ck.cocktail_kv16_attention(cache, turned, starts, max_new=max(piece), max_len=max(lens))
        done = [a + b for a, b in zip(done, piece)]
        row = 0
        for b, n in enumerate(piece):
            if n:
                at = torch.arange(done[b], device=dev)
                place = pages.table[b, at // 16].long()
                keys, values = (p[place, :, at % 16] for p in cache.pools)
                assert torch.equal(values, v[b][:done[b]])
                _check_turned(keys, k[b][:done[b]], np.arange(done[b]), _freq(d), False, 1.0, torch.float16)
                w, wl, mean_v, size = F.attention(_f64(turned[row:row + n]), _f64(keys), _f64(values))
                logit = 132 * 2.0 ** -24 * size + 2.0 ** -19
                assert (np.abs(_f64(out[row:row + n]) - w) <= 2.0 ** -11 * np.abs(w) + 2 * (2.0 ** -11 + logit + 400 * 2.0 ** -24)[..., None] * mean_v).all()
                row += n
    ck.cocktail_pages_check(pages)
    shape = ck.make_shape(2, hq, hkv, d, chunk, 32)
    ids = pages.table.long()
    flat = [[p[ids[b, torch.arange(lens[b], device=dev) // 16], :, torch.arange(lens[b], device=dev) % 16].transpose(0, 1).cpu().numpy() for p in cache.pools] for b in range(2)]
    last = torch.randn(2, hq, d, device=dev, dtype=torch.float16)
    over_pages, _ = ck.cocktail_kv16_attention(cache, last)
    for mixed in (False, True):
        bits = [rng.choice(np.array([16, 4, 2], np.uint8), n // chunk) if mixed else np.full(n // chunk, 16, np.uint8) for n in lens]
        plan = ck.cocktail_plan(shape, lens, np.concatenate(bits), ck.cocktail_default_workers(shape))
        packed = ck.PackedCache(plan, dev)
        ck.cocktail_reorder_quantize_paged(packed, *cache.pools, pages.table)
        got, _ = ck.cocktail_decode_attention(packed, last)
        want, _ = CO.decode_attention(last.cpu().numpy(), CO.reorder_quantize([f[0] for f in flat], [f[1] for f in flat], bits, chunk, 32))
        worst = max(np.abs(_f64(got[b, h]) - want[b, h]).max() / np.abs(want[b, h]).max() for b in range(2) for h in range(hq))
        assert worst <= 2e-3
        if not mixed:
            # the last query of each sequence sees all keys in both; 2e-3 of the largest channel on either side
            far = (got.double() - over_pages.double()).abs().amax(-1) / over_pages.double().abs().amax(-1)
            assert (far <= 4e-3).all()


def _model(vocab, dim, seed):
    """A toy of a model in binary64: what token t at position p of a history brings, and logits from a result of attention."""
    rng = np.random.default_rng(seed)
    return {"k": rng.standard_normal((vocab, dim)), "v": rng.standard_normal((vocab, dim)), "q": rng.standard_normal((vocab, dim)) * 2,
            "head": rng.standard_normal((dim, vocab)) * 2}


@gpu
def test_a_beam_search_over_pages():
    """Requests with several hypotheses over a model's one layer: room, rotated append, attention, selection, forks of the pages and reordering of the histories,
    step by step.  Every hypothesis' result is that of attention over its own history, and the selection is the oracle's on the logits of the step."""
    dev = torch.device("cuda:0")
    groups, beams, vocab, d, steps, eos, page = 3, 4, 97, 64, 24, 5, 16
    rows = groups * beams
    M = _model(vocab, d, 1)
    dt = torch.float16
    t = {x: torch.from_numpy(M[x]).to(dev, dt) for x in ("k", "v", "q")}
    head = torch.from_numpy(M["head"]).to(dev, torch.float32)
    pages = ck.PageTable(rows, 64, rows * 4, page, dev)
    cache = ck.Kv16Cache(pages, 1, d, dt)
    rot = _rotation(d, True)
    prompt = np.random.default_rng(2).integers(6, vocab, (groups, 7))
    history = torch.zeros(rows, 64, dtype=torch.int32, device=dev)
    history[:, :7] = torch.from_numpy(np.repeat(prompt, beams, 0).astype(np.int32)).to(dev)
    # prompts once, then forked to all hypotheses
    counts = [7 if r % beams == 0 else 0 for r in range(rows)]
    starts = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), device=dev)
    ids = torch.from_numpy(prompt.reshape(-1)).to(dev)
    ck.cocktail_pages_resize(pages, torch.tensor(counts, dtype=torch.int32, device=dev), cache.pools)
    ck.cocktail_kv16_append(cache, t["k"][ids][:, None], t["v"][ids][:, None], starts, rot)
    ck.cocktail_pages_fork(pages, torch.arange(rows, dtype=torch.int32, device=dev) // beams * beams)
    scores = torch.tensor([0.0] + [-math.inf] * (beams - 1), device=dev).repeat(groups)
    finished = torch.zeros(rows, dtype=torch.bool, device=dev)
    token = torch.from_numpy(prompt[:, -1]).to(dev).repeat_interleave(beams)
    one = torch.ones(rows, dtype=torch.int32, device=dev)
    position = 7
    # the last prompt token's query first, without a new key
    query = lambda tok: t["q"][tok][:, None]  # noqa: E731
    turned = torch.empty(rows, 1, d, dtype=dt, device=dev)
    same = 0
    for step in range(steps):
        if step:
            ck.cocktail_pages_resize(pages, one, cache.pools)
            turned = ck.cocktail_kv16_append(cache, t["k"][token][:, None], t["v"][token][:, None], rotation=rot, q=query(token))
            history[:, position] = token.int()
            position += 1
        else:
            turned.copy_(torch.from_numpy(O.rotate(_f64(query(token)), np.full(rows, 6), _freq(d), True)))
        out, _ = ck.cocktail_kv16_attention(cache, turned)
        # every hypothesis against its own history
        live = (scores > -math.inf).cpu().numpy()
        for r in range(rows):
            if live[r]:
                h = history[r, :position].cpu().numpy()
                keys = O.rotate(_f64(t["k"])[h][:, None], np.arange(position), _freq(d), True)
                w, _, mean_v, size = F.attention(_f64(turned[r:r + 1]), keys, _f64(t["v"])[h][:, None])
                # K rounded to fp16 after the rotation: half a step in every product of a logit
                assert (np.abs(_f64(out[r:r + 1]) - w) <= 2.0 ** -11 * np.abs(w) + 2 * (2.0 ** -11 + 2.0 ** -11 * size[..., None] + 2.0 ** -14) * mean_v).all(), (step, r)
        logits = out[:, 0].float() @ head
        want = O.select(logits.double().cpu().numpy(), scores.tolist(), beams, beams, eos, finished.tolist())
        source, tok, score, ended = ck.cocktail_beam_select(logits, scores, beams, eos=eos, finished=finished)
        assert np.array_equal(source.cpu().numpy(), want[0]) and np.array_equal(tok.cpu().numpy(), want[1]) and np.array_equal(ended.cpu().numpy(), want[3])
        assert (np.abs(score.double().cpu().numpy() - want[2]) <= 2.0 ** -20 + 2.0 ** -23 * np.abs(want[2])).all()
        source = source.view(-1)
        old = history.clone()
        ck.cocktail_pages_fork(pages, source)
        ck.cocktail_beam_reorder(source, [history])
        assert torch.equal(history, old[source.long()])
        scores, token, finished = score.view(-1), tok.view(-1).long(), ended.view(-1)
        same += int((source == torch.arange(rows, device=dev)).sum())
    ck.cocktail_pages_check(pages)
    assert pages.seq_lens.tolist() == [position] * rows and 0 < same < steps * rows


@gpu
def test_many_hypotheses_and_the_largest_vocabulary():
    rng = np.random.default_rng(21)
    logits = torch.randn(1 << 20, 9, device="cuda:0", dtype=torch.float16)
    scores = torch.randn(1 << 20, device="cuda:0")
    got = ck.cocktail_beam_select(logits, scores, 64, keep=8)
    for g in rng.integers(0, 1 << 14, 40):
        rows = slice(64 * int(g), 64 * int(g) + 64)
        want = O.select(logits[rows].double().cpu().numpy(), scores[rows].tolist(), 64, 8)
        assert np.array_equal(got[0][g].cpu().numpy() - 64 * g, want[0][0]) and np.array_equal(got[1][g].cpu().numpy(), want[1][0])
    logits = torch.randn(3, 1 << 24, device="cuda:0")
    logits[1, -1], logits[2, 0] = 40.0, 41.0
    scores = torch.tensor([-3.0, -2.0, -1.0], device="cuda:0")
    got = ck.cocktail_beam_select(logits, scores, 3, keep=64, eos=(1 << 24) - 1)
    want = O.select(logits.double().cpu().numpy(), scores.tolist(), 3, 64, (1 << 24) - 1)
    assert got[0][0, :2].tolist() == [2, 1] and got[1][0, :2].tolist() == [0, (1 << 24) - 1] and got[3][0, :3].tolist() == [False, True, False]
    # (values of 2^24 terms in binary64 sums of eight in binary32: 2^-20)
    assert np.abs(got[2].double().cpu().numpy() - want[2]).max() <= 2.0 ** -20 + 2.0 ** -24 * np.abs(want[2]).max()


@gpu
def test_the_bindings_refusals():
    B = Batch([40, 20], 2, 128, 16, torch.float16)
    x = torch.zeros(4, 2, 128, device=B.dev, dtype=torch.float16)
    for bad in (x.float(), x.bfloat16(), x.cpu(), x[:, :1], x[..., :64]):
        with pytest.raises(TypeError):
            ck.cocktail_kv16_append(B.cache, bad, x)
        with pytest.raises((TypeError, ck.CocktailError)):
            ck.cocktail_kv16_attention(B.cache, bad)
    with pytest.raises(ValueError):
        ck.cocktail_kv16_append(B.cache, x, x[:2])
    rot = _rotation(128)
    for more in (dict(q=x), dict(q=x[:2], rotation=rot), dict(q_out=x), dict(positions=torch.zeros(4, dtype=torch.int32, device=B.dev)),
                 dict(q=x, rotation=rot, q_out=x[:2]), dict(rotation=_rotation(256))):
        with pytest.raises((ValueError, ck.CocktailError)):
            ck.cocktail_kv16_append(B.cache, x, x, **more)
    for more in (dict(rotation=rot, positions=torch.zeros(4, device=B.dev)), dict(rotation=rot, positions=torch.zeros(3, dtype=torch.int32, device=B.dev)),
                 dict(starts=torch.zeros(2, dtype=torch.int32, device=B.dev)), dict(q=x[0], rotation=rot)):
        with pytest.raises(TypeError):
            ck.cocktail_kv16_append(B.cache, x, x, **more)
    for bad in (torch.zeros(8, dtype=torch.float32, device=B.dev), torch.zeros(8, dtype=torch.float64), torch.zeros(4, 2, dtype=torch.float64, device=B.dev)):
        with pytest.raises(TypeError):
            ck.Rotation(bad)
    with pytest.raises(TypeError):
        ck.Kv16Cache(B.pages, 2, 128, torch.float32)
    with pytest.raises(TypeError):
        ck.Kv16Cache(B.pages, 2, 128, torch.bfloat16, pools=B.cache.pools)
    with pytest.raises(ValueError):
        ck.Kv16Cache(B.pages, 2, 128, pools=(B.cache.k, B.cache.k))
    with pytest.raises(ck.CocktailError):
        ck.Kv16Cache(B.pages, 2, 96)
    with pytest.raises(ValueError):
        ck.cocktail_kv16_attention(B.cache, x, out=x[:2])
    with pytest.raises(ValueError):
        ck.cocktail_kv16_attention(B.cache, x, lse=torch.zeros(4, 2, device=B.dev, dtype=torch.float16))
    logits, scores = torch.zeros(4, 10, device=B.dev), torch.zeros(4, device=B.dev)
    for args in ((logits.double(), scores, 2), (logits[0], scores, 2), (logits.t(), scores, 2), (logits, scores[:2], 2), (logits, scores.half(), 2),
                 (logits, scores.cpu(), 2)):
        with pytest.raises(TypeError):
            ck.cocktail_beam_select(*args)
    for beams in (0, 3, -1):
        with pytest.raises(ValueError):
            ck.cocktail_beam_select(logits, scores, beams)
    with pytest.raises(ck.CocktailError):
        ck.cocktail_beam_select(logits, scores, 2, keep=65)
    with pytest.raises(ck.CocktailError):
        ck.cocktail_beam_select(logits, scores, 2, finished=torch.zeros(4, dtype=torch.bool, device=B.dev))        # no eos
    # nothing to do
    empty = torch.zeros(0, 2, 128, device=B.dev, dtype=torch.float16)
    starts = torch.zeros(3, dtype=torch.int32, device=B.dev)
    assert ck.cocktail_kv16_append(B.cache, empty, empty, starts) is None
    out, lse = ck.cocktail_kv16_attention(B.cache, empty, starts)
    assert out.shape == (0, 2, 128) and lse.shape == (0, 2)
    assert ck.cocktail_beam_reorder(starts, []) == []


# ---- memory that results share with arguments ----------------------------------------------------------------------------------------


def test_results_that_overlap_with_arguments_are_refused():
    L = _lib.lib()
    pages = _lib.PageTableDesc(4096, 4096, 4096, 4096, 4, 8, 16, 32)
    cache = C.byref(_lib.Kv16CacheDesc(pages, 1 << 30, 1 << 31, 2, 128, _lib.FP16, 0))
    turn = C.byref(_lib.RotationDesc(4096, 128, 0, 1.0, 0))
    k, v, q = 1 << 20, 2 << 20, 3 << 20                       # eight rows of two heads, and of four that lie a row of eight apart

    def append(q_out, **more):
        a = dict(q=q, st=1024, sh=128)
        a.update(more)
        return L.cocktail_kv16_append(cache, k, v, 256, 128, 8, 4096, turn, None, a["q"], 4, a["st"], a["sh"], q_out, None)

    def attention(out, st=1024):
        return L.cocktail_kv16_attention(cache, 4, q, st, 128, 8, 4096, 8, 0, 0.0, out, None, 4096, 1 << 40, None)
    last = q + 2 * (7 * 1024 + 4 * 128) - 16                  # the last sixteen bytes of the queries
    for call, where in [(append, x) for x in (q, q + 16, last, q - 2 * 8 * 512 + 16, k, k + 2 * 8 * 256 - 16, v, v - 2 * 8 * 512 + 16)] + \
            [(attention, x) for x in (q, q + 16, last, q - 2 * 8 * 512 + 16)]:
        assert call(where) == _lib.EINVAL, (call, where - q)
        assert b"over" in L.cocktail_last_error() or b"in place" in L.cocktail_last_error()
    assert append(k, q=k, st=512) == _lib.EINVAL and b"over" in L.cocktail_last_error()
    assert attention(q + 512 * 2, st=512) == _lib.EINVAL and b"over" in L.cocktail_last_error()

    def select(keep=4, **more):
        a = dict(logits=1 << 20, scores=1 << 16, finished=1 << 17, source=1 << 12, token=2 << 12, score=3 << 12, out=4 << 12)
        a.update(more)
        return L.cocktail_beam_select(a["logits"], _lib.FP32, 128, 2, 4, 100, keep, a["scores"], a["finished"], 7, a["source"], a["token"], a["score"], a["out"],
                                      1 << 28, 1 << 40, None)
    logits_end = (1 << 20) + 4 * (7 * 128 + 100)
    for more in (dict(source=2 << 12), dict(source=(2 << 12) + 28), dict(token=3 << 12), dict(score=(4 << 12) - 28), dict(out=(1 << 12) + 31),
                 dict(source=1 << 20), dict(token=logits_end - 4), dict(score=(1 << 20) - 28), dict(out=logits_end - 1), dict(source=1 << 16),
                 dict(score=(1 << 16) + 4), dict(score=1 << 17), dict(out=1 << 16), dict(out=(1 << 17) + 1), dict(token=(1 << 17) + 4),
                 dict(score=1 << 16, finished=(1 << 16) + 4)):
        assert select(**more) == _lib.EINVAL, more
        assert b"overlap" in L.cocktail_last_error(), more


def test_more_rows_than_a_launch_takes_are_refused():
    L = _lib.lib()
    pages = _lib.PageTableDesc(4096, 4096, 4096, 4096, 4096, 1, 16, 4096)
    cache = C.byref(_lib.Kv16CacheDesc(pages, 1 << 40, 1 << 41, 1024, 128, _lib.FP16, 0))
    assert L.cocktail_kv16_attention(cache, 1024, 1 << 42, 1024 * 128, 128, 1 << 18, 4096, 64, 0, 0.0, 1 << 43, None, 1 << 44, 1 << 44, None) == _lib.EINVAL
    assert b"too many" in L.cocktail_last_error()


@gpu
def test_queries_of_no_tokens():
    B = Batch([40, 20], 2, 128, 16, torch.float16)
    empty = torch.zeros(0, 2, 128, device=B.dev, dtype=torch.float16)
    starts = torch.zeros(3, dtype=torch.int32, device=B.dev)
    before = [t.clone() for t in B.cache.pools]
    for given in (None, empty.clone()):
        got = ck.cocktail_kv16_append(B.cache, empty, empty, starts, _rotation(128), empty, q_out=given)
        assert got.shape == (0, 2, 128) and (given is None or got is given)
    assert all(torch.equal(t.view(torch.int16), u.view(torch.int16)) for t, u in zip(B.cache.pools, before))


@gpu
@pytest.mark.parametrize("lens, new, rep, max_len", [
    ([300, 40, 7], [1, 1, 1], 4, 300),             # a workgroup per segment
    ([9000, 40, 2500], [1, 1, 1], 4, 0),           # cut by tokens, states joined
    ([700, 3000], [6, 9], 4, 0),
    ([900, 300, 130], [900, 1, 130], 4, 0),        # both kernels
    ([5000], [200], 2, 0),                         # many rows, their keys in parts
    ([700, 700], [700, 700], 1, 700),
    ([900, 31, 2000, 64, 500, 1, 333, 1200], [9] * 8, 4, 0),     # shares of workgroups
    ([100, 31, 200, 64], [9] * 4, 4, 200),         # a workgroup per segment, 36 rows
])
def test_attention_in_place(lens, new, rep, max_len):
    B = Batch(lens, 2, 128, 16, torch.float16, seed=5)
    for t in B.cache.pools:
        t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(3)).to(t.dtype))
    q = torch.randn(sum(new), 2 * rep, 128, generator=torch.Generator().manual_seed(4)).to(B.dev, torch.float16)
    starts = torch.tensor([0, *np.cumsum(new)], dtype=torch.int32, device=B.dev)
    want, lse = ck.cocktail_kv16_attention(B.cache, q, starts, max(new), max_len)
    own = q.clone()
    got, again = ck.cocktail_kv16_attention(B.cache, own, starts, max(new), max_len, out=own)
    assert got is own and torch.equal(got, want) and torch.equal(again, lse)


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("lens, new, kv_heads, rep, d, page", [
    ([9001], [1], 1, 2, 128, 16),
    ([33, 20011, 700], [1, 1, 1], 1, 3, 64, 16),
    ([12345, 9000], [1, 1], 1, 8, 128, 48),
    ([4096, 4192, 4096], [1, 1, 1], 1, 1, 128, 64),                # segments that end where workgroups do, and a wave before
    ([5000, 0, 4097], [9, 3, 7], 2, 4, 128, 16),                   # states of 48 rows
    ([2048], [16], 1, 4, 64, 16),                                  # of 64
    ([3000, 777], [5, 6], 1, 5, 128, 32),                          # of 32
    ([6000 if b in (3, 40, 99) else 10 for b in range(100)], [1 if b in (3, 40, 99) else 0 for b in range(100)], 1, 4, 128, 16),
    ([30000, 40, 30016], [1, 1, 1], 4, 4, 64, 16),
])
def test_workgroups_that_leave_one_state(lens, new, kv_heads, rep, d, page, dtype):
    B = Batch(lens, kv_heads, d, page, DTYPES[dtype], seed=len(lens), spread=4.0)
    B.store_all()
    q = B.query(new, rep)
    for max_len in (max(lens), 0, max(lens) // 3):                 # (other numbers of workers)
        out, lse = ck.cocktail_kv16_attention(B.cache, q, B.starts(new), max(new), max_len)
        B.check(q, new, out, lse)
        again, lse2 = ck.cocktail_kv16_attention(B.cache, q, B.starts(new), max(new), max_len)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("num_seqs, kv_heads, rep, new, longest, d, page", [
    (40, 2, 8, 8, 900, 128, 16),         # 64 rows
    (40, 1, 8, 6, 1300, 128, 48),        # 48
    (33, 4, 5, 6, 500, 64, 16),          # 30
    (130, 1, 16, 4, 300, 64, 32),        # more sequences than lanes
    (70, 2, 12, 2, 700, 128, 16),        # 24
    (3, 8, 16, 3, 4000, 128, 16),
    (600, 1, 3, 7, 60, 64, 16),
])
def test_several_queries_of_many_sequences(num_seqs, kv_heads, rep, new, longest, d, page, dtype):
    rng = np.random.default_rng(num_seqs)
    lens = [int(t) for t in rng.integers(0, longest + 1, num_seqs)]
    lens[0], lens[-1] = longest, 0
    count = [int(n) for n in rng.integers(0, new + 1, num_seqs)]
    count[0] = count[-1] = new
    B = Batch(lens, kv_heads, d, page, DTYPES[dtype], seed=num_seqs, spread=4.0)
    B.store_all()
    q = B.query(count, rep)
    for max_len in (longest, 0, 1, 20000):                         # a workgroup per segment, shares of waves or of workgroups
        out, lse = ck.cocktail_kv16_attention(B.cache, q, B.starts(count), new, max_len)
        B.check(q, count, out, lse)
        again, lse2 = ck.cocktail_kv16_attention(B.cache, q, B.starts(count), new, max_len)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
