"""Memory that results of the paged 16-bit cache and of beam search share with each other or with what a call reads: refused before anything is launched,
also where only a few bytes are shared; what lies side by side is not."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck
from paper_2503_23294_amd import _lib
from test_kv16 import Batch
from test_kv16_edges import quiet  # noqa: F401 (a fixture)

gpu = pytest.mark.gpu
MB = 1 << 20


def _overlap_refused(rc, what):
    assert rc == _lib.EINVAL, what
    message = _lib.lib().cocktail_last_error()
    assert b"overlap" in message or b"in place only" in message, (what, message)      # (exactly over rows that lie apart)


# where things are, and their bytes: four sequences of up to eight pages of sixteen tokens, 32 pages of 2 heads of 128 channels, eight rows of four heads
PLACES = dict(table=(MB, 4 * 4 * 8), seq_lens=(2 * MB, 4 * 4), status=(3 * MB, 16), k=(4 * MB, 32 * 2 * 16 * 256), v=(6 * MB, 32 * 2 * 16 * 256), starts=(8 * MB, 4 * 5),
              q=(9 * MB, 2 * (7 * 1024 + 4 * 128)))


def _cache(**more):
    at = {n: p[0] for n, p in PLACES.items()}
    at.update(more)
    pages = _lib.PageTableDesc(at["table"], at["seq_lens"], 20 * MB, at["status"], 4, 8, 16, 32)
    return C.byref(_lib.Kv16CacheDesc(pages, at["k"], at["v"], 2, 128, _lib.FP16, 0))


def _ends(place, size, align):
    """Addresses of `size` bytes that share a few with a place: its beginning, and its end."""
    at, n = place
    return [at - size + align, at, at + (n - 1) // align * align]


def test_results_of_attention_over_what_the_call_reads():
    L = _lib.lib()
    need = C.c_size_t(0)
    assert L.cocktail_kv16_attention_workspace(_cache(), 4, 8, 8, 0, 0, C.byref(need)) == 0

    def call(out=10 * MB, lse=11 * MB, ws=12 * MB, st=1024):
        return L.cocktail_kv16_attention(_cache(), 4, PLACES["q"][0], st, 128, 8, PLACES["starts"][0], 8, 0, 0.0, out, lse, ws, need.value, None)
    out_bytes, lse_bytes = 8 * 512 * 2, 8 * 4 * 4
    for name in ("q", "k", "v", "table", "seq_lens", "starts"):
        for at in _ends(PLACES[name], lse_bytes, 4):
            _overlap_refused(call(lse=at), ("lse", name, at))
        for at in _ends(PLACES[name], out_bytes, 16):
            _overlap_refused(call(out=at), ("out", name, at))
        for at in _ends(PLACES[name], need.value // 16 * 16, 16):
            _overlap_refused(call(ws=at), ("workspace", name, at))
    for at in _ends((10 * MB, out_bytes), lse_bytes, 4):
        _overlap_refused(call(lse=at), ("lse", "out", at))
    for at in _ends((12 * MB, need.value), lse_bytes, 4):
        _overlap_refused(call(lse=at), ("lse", "workspace", at))
    for at in _ends((12 * MB, need.value), out_bytes, 16):
        _overlap_refused(call(out=at), ("out", "workspace", at))
    # in place: the log-sum-exp is elsewhere all the same
    _overlap_refused(call(out=PLACES["q"][0], lse=PLACES["q"][0] + 512, st=512), "in place")


def test_queries_of_append_over_what_the_call_reads_or_stores_to():
    L = _lib.lib()
    rows = dict(PLACES, k_rows=(13 * MB, 8 * 256 * 2), v_rows=(14 * MB, 8 * 256 * 2), positions=(15 * MB, 4 * 8), inv_freq=(16 * MB, 8 * 64))
    turn = C.byref(_lib.RotationDesc(rows["inv_freq"][0], 128, 0, 1.0, 0))

    def call(q_out=10 * MB, st=1024, cache=None):
        return L.cocktail_kv16_append(cache or _cache(), rows["k_rows"][0], rows["v_rows"][0], 256, 128, 8, rows["starts"][0], turn, rows["positions"][0],
                                      rows["q"][0], 4, st, 128, q_out, None)
    for name in rows:
        for at in _ends(rows[name], 8 * 512 * 2, 16):
            _overlap_refused(call(at), (name, at))


def test_pools_that_share_memory():
    """K and V of a token would be stored over each other."""
    L = _lib.lib()
    k, n = PLACES["k"]
    for v in _ends((k, n), n, 16):
        _overlap_refused(L.cocktail_kv16_append(_cache(v=v), 13 * MB, 14 * MB, 256, 128, 8, PLACES["starts"][0], None, None, None, 0, 0, 0, None, None), v)


@gpu
def test_a_cache_of_pools_that_share_memory():
    B = Batch([40, 9], 2, 64, 16, torch.float16)
    flat = torch.zeros(2 * B.cache.k.numel(), dtype=torch.float16, device=B.dev)
    n = B.cache.k.numel()
    at = lambda first: flat[first:first + n].view(B.cache.k.shape)  # noqa: E731
    for k, v in ((0, 0), (0, n - 8), (n - 8, 0), (8, 0)):
        with pytest.raises(ValueError):
            ck.Kv16Cache(B.pages, 2, 64, pools=(at(k), at(v)))
    for k, v in ((0, n), (n, 0)):
        ck.Kv16Cache(B.pages, 2, 64, pools=(at(k), at(v)))


def _carved(dev, *specs):
    """Tensors side by side in one allocation, sixteen bytes aligned each where their sizes are."""
    sizes = [int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size() for shape, dtype in specs]
    flat = torch.zeros(sum(sizes), dtype=torch.uint8, device=dev)
    out, at = [], 0
    for (shape, dtype), n in zip(specs, sizes):
        out.append(flat[at:at + n].view(dtype).view(shape))
        at += n
    return out


@gpu
@pytest.mark.parametrize("new", [1, 40])
def test_attention_between_its_neighbours(new):
    """q, out, lse and both pools without a byte between them; and the calls that are refused leave everything as it is."""
    B = Batch([300, 77], 2, 128, 16, torch.float16, seed=new)
    B.store_all()
    q = B.query([new, new], 4)
    want, wlse = ck.cocktail_kv16_attention(B.cache, q)
    f16 = torch.float16
    k, own, out, lse, v = _carved(B.dev, (B.cache.k.shape, f16), (q.shape, f16), (q.shape, f16), (wlse.shape, torch.float32), (B.cache.v.shape, f16))
    for to, of in ((k, B.cache.k), (own, q), (v, B.cache.v)):
        to.view(torch.int16).copy_(of.view(torch.int16))
    cache = ck.Kv16Cache(B.pages, 2, 128, pools=(k, v))
    ck.cocktail_kv16_attention(cache, own, out=out, lse=lse)
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    kept = [t.view(torch.int16).clone() for t in (k, own, v)]
    over = lambda t: t.view(-1)[:q.numel()].view(q.shape)  # noqa: E731
    floats = lambda t: t.view(-1)[:2 * wlse.numel()].view(torch.float32).view(wlse.shape)  # noqa: E731
    for more in (dict(lse=floats(own)), dict(lse=floats(out), out=out), dict(lse=floats(k)), dict(lse=floats(v)), dict(out=over(k)), dict(out=over(v)),
                 dict(out=own, lse=floats(own))):
        with pytest.raises(ck.CocktailError, match="overlap"):
            ck.cocktail_kv16_attention(cache, own, **more)
    assert torch.equal(out, want) and all(torch.equal(t.view(torch.int16), old) for t, old in zip((k, own, v), kept))


@gpu
def test_append_between_its_neighbours():
    B = Batch([40, 9], 2, 64, 16, torch.float16, seed=3)
    q = B.query([40, 9], 3)
    rot = ck.Rotation(torch.full((32,), 0.1, dtype=torch.float64, device=B.dev))
    want = ck.cocktail_kv16_append(B.cache, B.k, B.v, B.starts([40, 9]), rotation=rot, q=q)
    f16 = torch.float16
    k, q_out, v, rows_k, own, rows_v, _ = _carved(B.dev, *((t.shape, f16) for t in (B.cache.k, q, B.cache.v, B.k, q, B.v, q)))
    rows_k.copy_(B.k), own.copy_(q), rows_v.copy_(B.v)
    for to, of in ((k, B.cache.k), (v, B.cache.v)):
        to.view(torch.int16).copy_(of.view(torch.int16))
    cache = ck.Kv16Cache(B.pages, 2, 64, pools=(k, v))
    ck.cocktail_kv16_append(cache, rows_k, rows_v, B.starts([40, 9]), rotation=rot, q=own, q_out=q_out)
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    assert same(q_out, want) and same(k, B.cache.k) and same(v, B.cache.v) and same(rows_k, B.k) and same(rows_v, B.v) and same(own, q)
    kept = [t.clone() for t in (k, v, rows_k, own, rows_v)]
    for place in (k, v, rows_k, rows_v, own):
        start = place.storage_offset()
        room = k.as_strided(q.shape, q.stride(), max(0, start - 8))
        with pytest.raises(ck.CocktailError, match="overlap"):
            ck.cocktail_kv16_append(cache, rows_k, rows_v, B.starts([40, 9]), rotation=rot, q=own, q_out=room)
    assert all(same(t, old) for t, old in zip((k, v, rows_k, own, rows_v), kept))
    assert ck.cocktail_kv16_append(cache, rows_k, rows_v, B.starts([40, 9]), rotation=rot, q=own, q_out=own) is own and same(own, want)


def test_the_workspace_of_a_selection():
    L = _lib.lib()
    need = C.c_size_t(0)
    assert L.cocktail_beam_select_workspace(2, 4, 100, 4, C.byref(need)) == 0
    places = dict(logits=(MB, 4 * (7 * 128 + 100)), scores=(2 * MB, 32), finished=(3 * MB, 8), source=(4 * MB, 32), token=(5 * MB, 32), score=(6 * MB, 32),
                  out=(7 * MB, 8))
    p = {n: at for n, (at, _) in places.items()}
    for name in places:
        for ws in _ends(places[name], need.value // 16 * 16, 16):
            _overlap_refused(L.cocktail_beam_select(p["logits"], _lib.FP32, 128, 2, 4, 100, 4, p["scores"], p["finished"], 7, p["source"], p["token"], p["score"],
                                                    p["out"], ws, need.value, None), (name, ws))


# ---- reordering --------------------------------------------------------------------------------------------------------------------


def _reorder(states, source=MB, rows=4):
    """states: (from, to, bytes of a row)"""
    n = len(states)
    of, to, size = zip(*states)
    return _lib.lib().cocktail_beam_reorder(source, rows, (C.c_void_p * n)(*of), (C.c_void_p * n)(*to), (C.c_int64 * n)(*size), n, None)


@pytest.mark.parametrize("states", [
    [(MB, MB, 4)],                                          # in place, the sources themselves
    [(MB - 60, MB - 60, 16)], [(MB + 12, MB + 12, 16)],     # or the last or first word of them
    [(2 * MB, MB, 4)], [(2 * MB, MB + 15, 1)], [(2 * MB, MB - 3, 1)],
    [(3 * MB, 3 * MB, 8), (2 * MB, MB + 8, 64)],
])
def test_states_that_are_written_over_the_sources(states):
    _overlap_refused(_reorder(states), states)


@pytest.mark.parametrize("states", [
    [(2 * MB, 2 * MB, 16), (2 * MB, 2 * MB, 16)],           # written twice, in place and not
    [(2 * MB, 2 * MB, 16), (2 * MB + 63, 2 * MB + 63, 1)],
    [(2 * MB, 3 * MB, 16), (4 * MB, 3 * MB + 60, 32)],
    [(2 * MB, 3 * MB, 16), (3 * MB - 4, 3 * MB - 4, 2)],
    [(2 * MB, 2 * MB + 16, 16)],                            # read and written
    [(2 * MB, 2 * MB - 63, 16)],
    [(2 * MB, 3 * MB, 16), (3 * MB, 4 * MB, 16)],
    [(2 * MB, 3 * MB, 16), (3 * MB - 124, 4 * MB, 32)],
    [(5 * MB, 6 * MB, 1), (2 * MB, 3 * MB, 16), (7 * MB, 8 * MB, 4), (9 * MB, 9 * MB, 64), (9 * MB, 2 * MB + 32, 4)],
])
def test_states_that_are_written_over_each_other(states):
    for order in (states, states[::-1]):
        _overlap_refused(_reorder(order), order)


def test_states_that_are_views_of_the_sources(quiet):
    source = torch.zeros(12, dtype=torch.int32)
    state = torch.zeros(4, 6)
    for states, out in (([source[:4]], None), ([state, source[:8].view(4, 2)], None), ([torch.zeros(4, 1)], [source[:4].view(torch.float32).view(4, 1)]),
                        ([torch.zeros(4, 2, dtype=torch.int32)], [source[3:11].view(4, 2)])):
        with pytest.raises(ValueError):
            ck.cocktail_beam_reorder(source[:4], states, out=out)
    ck.cocktail_beam_reorder(source[:4], [source[4:8]])                                    # next to them
    ck.cocktail_beam_reorder(source[:4], [source[:4]], out=[source[4:8]])                  # read twice


@gpu
def test_states_next_to_the_sources():
    """A state that ends where the sources begin, and one that begins where they end; a history to which the sources themselves are copied."""
    rows = 300
    flat = torch.arange(6 * rows, dtype=torch.int32, device="cuda:0")
    source = flat[2 * rows:3 * rows]
    source.copy_(torch.arange(rows, device="cuda:0").flip(0))
    want = flat.clone()
    a, b, copy = flat[:2 * rows].view(rows, 2), flat[3 * rows:4 * rows], flat[4 * rows:5 * rows]
    ck.cocktail_beam_reorder(source, [a, b])
    ck.cocktail_beam_reorder(source, [source], out=[copy])
    order = source.long()
    want[:2 * rows] = want[:2 * rows].view(rows, 2)[order].view(-1)
    want[3 * rows:4 * rows] = want[3 * rows:4 * rows][order]
    want[4 * rows:5 * rows] = source[order]
    assert torch.equal(flat, want)
    with pytest.raises(ValueError):
        ck.cocktail_beam_reorder(source, [flat[rows:2 * rows + 1][1:], flat[2 * rows + 1:3 * rows + 1]])
    assert torch.equal(flat, want)


@gpu
def test_a_state_that_is_copied_and_then_reordered_in_place():
    """By the C entry: the copy has what the state was before the call."""
    rows, dev = 50, "cuda:0"
    rng = np.random.default_rng(1)
    flat = torch.from_numpy(rng.integers(0, 1 << 30, 3 * rows * 700)).to(dev, torch.int32).view(3, rows, 700)
    source = torch.from_numpy(rng.integers(0, rows, rows)).to(dev, torch.int32)
    want = flat.clone()
    want[0] = want[1] = flat[1][source.long()]
    a, b = flat[0].data_ptr(), flat[1].data_ptr()
    assert _lib.lib().cocktail_beam_reorder(source.data_ptr(), rows, (C.c_void_p * 2)(b, b), (C.c_void_p * 2)(a, b), (C.c_int64 * 2)(2800, 2800), 2,
                                            torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(flat, want)


def test_reordering_of_no_rows_is_refused(quiet):
    none = torch.zeros(0, dtype=torch.int32)
    for states, out in (([torch.zeros(0, 3)], None), ([torch.zeros(0, 3)], [torch.zeros(0, 3)]), ([], None)):
        with pytest.raises(ValueError):
            ck.cocktail_beam_reorder(none, states, out=out)
