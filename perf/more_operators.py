"""The operators of the paged 16-bit cache and of beam search as timed cases: new tokens are rotated by their position and appended to
16-bit pages, the newest tokens of every sequence attend to those pages, and a step of beam search selects the best continuations and
reorders what its beams carry.

A case is a dict of plain values:
  kind       "append" (K of new tokens is rotated and stored with V, their queries are rotated too), "attend" (attention of every sequence's
             newest tokens over the pages), "beam" (selection over beams and vocabulary, and reordering of states)
  dtype      of K, V and q, or of the logits: float16, bfloat16, float32 (logits only)
append and attend:
  batch, q_heads, kv_heads, head_dim, page     sequences, heads, channels, tokens per page
  tokens     tokens of the longest sequence, the new ones included; shortest: of the shortest one
  new        new tokens of the sequence that has most; fewest: of the one that has fewest
  lengths    which lengths a ragged batch has between the two
  rotary     channels of a head that are rotated (append); interleaved: neighbours are pairs, else channels half of them apart
  base       of the geometric row of angles a token advances by
beam:
  groups, beams, vocab     requests, hypotheses of each, tokens to choose from
  keep       continuations that are selected for each request
  first      the first step of a search: all beams but one are without a probability
  ended      share of the beams (in percent) that have ended before
  history    tokens that every beam carries (int32), state: 16-bit values that it carries, as a layer with a recurrent state has
  layers     tensors of such values

K, V, q and logits are Gaussian (logits with a spread of three, and some tokens of every row raised as a model that knows what it wants does);
pages lie in random order in a pool whose unused places hold the values of sequences that are gone.
"""
import math
import random

import torch

own = False

EOS = 2


def _paged(name, kind, batch, q_heads, kv_heads, tokens, new, **more):
    case = {"name": name, "kind": kind, "dtype": "float16", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": 128,
            "page": 64, "tokens": tokens, "shortest": tokens, "new": new, "fewest": new, "lengths": 0, "rotary": 128, "interleaved": False,
            "base": 10000.0}
    case.update(more)
    return case


def _beam(name, groups, beams, vocab, **more):
    case = {"name": name, "kind": "beam", "dtype": "float32", "groups": groups, "beams": beams, "vocab": vocab, "keep": beams, "first": False,
            "ended": 0, "history": 128, "state": 0, "layers": 0}
    case.update(more)
    return case


def listed():
    return [
        # a step of a running batch: one generated token per sequence, far into its context
        _paged("append_step_b8", "append", 8, 32, 8, 16384, 1, shortest=4099, lengths=1, page=16, base=500000.0),
        # prompts of unlike, odd lengths, bfloat16, 64 channels a head of which half are rotated, neighbours in pairs
        _paged("append_ragged_bf16_d64_b6", "append", 6, 16, 16, 16001, 16001, shortest=37, fewest=37, lengths=2, page=16, dtype="bfloat16",
               head_dim=64, rotary=32, interleaved=True),
        # the whole prompt of a grouped-query layer
        _paged("append_prompt_32k_gqa4", "append", 1, 32, 8, 32768, 32768, base=500000.0),
        # a short context on few heads: launches and latency
        _paged("decode_2k_8h", "attend", 1, 8, 8, 2048, 1),
        # a grouped-query layer serving eight requests of unlike, odd lengths
        _paged("decode_ragged_gqa4_b8", "attend", 8, 32, 8, 130001, 1, shortest=8193, lengths=5, page=16),
        # a full batch of a large layer, eight query heads per kv head
        _paged("decode_4k_gqa8_bf16_b64", "attend", 64, 64, 8, 4097, 1, shortest=512, lengths=6, page=32, dtype="bfloat16"),
        # drafts of one to six tokens are verified against 16K contexts
        _paged("verify_16k_gqa8_b8", "attend", 8, 64, 8, 16390, 6, shortest=9001, fewest=1, lengths=7, page=16),
        # a chunk of a long prompt: 2048 new tokens behind 30K
        _paged("chunk_2k_of_32k_gqa4", "attend", 1, 32, 8, 32768, 2048),
        # whole prompts: the most arithmetic
        _paged("prompt_8k_32h_bf16", "attend", 2, 32, 32, 8190, 8190, shortest=4095, fewest=4095, lengths=8, dtype="bfloat16"),
        # one request with four hypotheses: latency
        _beam("beam_1x4_32k", 1, 4, 32000),
        # eight requests with eight each, odd vocabulary, some hypotheses have ended
        _beam("beam_8x8_bf16", 8, 8, 65001, dtype="bfloat16", ended=20, history=701, state=8192, layers=4),
        # a full batch over a large vocabulary, with the recurrent states of some layers
        _beam("beam_64x8_bf16", 64, 8, 131072, dtype="bfloat16", ended=10, history=1024, state=65536, layers=2),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "append", "decode", "decode", "decode", "verify", "verify", "chunk", "prompt", "beam", "beam", "beam"])
    if kind == "beam":
        beams = rng.choice([1, 2, 3, 4, 4, 5, 8, 8, 16, 32])
        groups = _log_uniform(rng, 1, 64)
        vocab = _log_uniform(rng, 1000, min(262144, 64 * 8 * 131072 // (groups * beams)))
        keep = rng.choice([beams, beams, beams, min(64, 2 * beams)])
        carried = keep == beams
        layers = rng.choice([0, 1, 3]) if carried else 0
        return {"kind": "beam", "dtype": rng.choice(["float32", "float16", "bfloat16"]), "groups": groups, "beams": beams, "vocab": vocab,
                "keep": keep, "first": rng.random() < 0.15, "ended": rng.choice([0, 0, 10, 40]),
                "history": _log_uniform(rng, 1, 2048) if carried else 0, "state": 8 * _log_uniform(rng, 1, 4096) if layers else 0, "layers": layers}
    page = rng.choice([16, 16, 32, 48, 64, 128, 256])
    head_dim = rng.choice([128, 128, 128, 64])
    dtype = rng.choice(["float16", "bfloat16"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 8, 16, 32, 40])
    rep = rng.choice([1, 1, 2, 3, 4, 4, 5, 7, 8, 8, 12, 16]) if kv_heads <= 8 else rng.choice([1, 1, 2])
    batch = rng.choice([1, 1, 2, 3, 5, 8, 24])
    rows = 8 * 8 * 65536 * 128 // (kv_heads * head_dim)           # about as many keys as the largest listed case has
    if kind == "append":
        tokens = _log_uniform(rng, 1, min(131072, max(1, rows // batch)))
        most = 32768 * 48 * 128 // (kv_heads * (rep + 2) * head_dim * batch)
        new = _log_uniform(rng, 1, max(1, min(tokens, most)))
    elif kind == "decode":
        tokens, new = _log_uniform(rng, 200, min(131072, rows // batch)), 1
    elif kind == "verify":
        new = rng.randint(2, 16)
        tokens = _log_uniform(rng, 200, min(65536, rows // batch))
    else:
        # no more products than the listed prompts have
        batch = rng.choice([1, 1, 2, 3])
        most = 2 * 32 * 8190 * 8190 // (kv_heads * rep * batch) // 4
        tokens = _log_uniform(rng, 300, min(16384, int(math.sqrt(most)) if kind == "prompt" else 16384))
        new = tokens if kind == "prompt" else max(17, min(tokens // rng.randint(2, 8), most // tokens))
    ragged = batch > 1 and rng.random() < 0.6
    shortest = max(1, _log_uniform(rng, max(1, tokens // 16), tokens)) if ragged else tokens
    fewest = max(1, min(new, shortest) // rng.randint(1, 4)) if ragged else new
    return {"kind": "append" if kind == "append" else "attend", "dtype": dtype, "batch": batch, "q_heads": kv_heads * rep, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "tokens": tokens, "shortest": shortest, "new": min(new, tokens), "fewest": min(fewest, new, tokens),
            "lengths": rng.randrange(1000), "rotary": rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4]),
            "interleaved": rng.random() < 0.4, "base": rng.choice([10000.0, 500000.0, 1000000.0])}


# ---- what a case looks like ----------------------------------------------------------------------------------------------


def _ragged(rng, n, longest, shortest):
    inner = [rng.randint(shortest, longest) for _ in range(n)]
    seqs = ([longest, shortest] + inner)[:n]
    rng.shuffle(seqs)
    return seqs


def _lengths(case):
    """Tokens of every sequence, and how many of them are new."""
    rng = random.Random(case["lengths"])
    lens = _ragged(rng, case["batch"], case["tokens"], case["shortest"])
    if case["new"] == case["tokens"]:
        return lens, list(lens)
    new = _ragged(rng, case["batch"], case["new"], case["fewest"])
    return lens, [min(a, b) for a, b in zip(lens, new)]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 31)


def _dtype(case):
    return getattr(torch, case["dtype"])


def _prefix(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _normal(gen, shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)


def _cache_state(case, seed):
    """Table, lengths and both pools [pages, heads, page, D]; every place holds a value, of a sequence or of one that is gone."""
    gen = _generator(seed)
    lens, new = _lengths(case)
    p = case["page"]
    need = [-(-t // p) for t in lens]
    pages = sum(need) + 3
    ids = torch.rand(pages, device="cuda", generator=gen).argsort().int()
    table = torch.full((case["batch"], max(need) + 1), -1, dtype=torch.int32, device="cuda")
    cols = torch.arange(table.shape[1], device="cuda")
    table[cols < torch.tensor(need, device="cuda")[:, None]] = ids[:sum(need)]
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[ids[:sum(need)].long()] = 1
    shape = (pages, case["kv_heads"], p, case["head_dim"])
    state = {"case": case, "table": table, "refs": refs, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"),
             "starts": torch.tensor(_prefix(new), dtype=torch.int32, device="cuda"),
             "pool_k": _normal(gen, shape, _dtype(case)), "pool_v": _normal(gen, shape, _dtype(case))}
    total = sum(new)
    if case["kind"] == "append":
        state["k"] = _normal(gen, (total, case["kv_heads"], case["head_dim"]), _dtype(case))
        state["v"] = _normal(gen, (total, case["kv_heads"], case["head_dim"]), _dtype(case))
        r = case["rotary"]
        state["inv_freq"] = torch.tensor([case["base"] ** (-2.0 * i / r) for i in range(r // 2)], dtype=torch.float64, device="cuda")
    state["q"] = _normal(gen, (total, case["q_heads"], case["head_dim"]), _dtype(case))
    return state


def _beam_state(case, seed):
    gen = _generator(seed)
    g, b, v = case["groups"], case["beams"], case["vocab"]
    rows = g * b
    logits = torch.empty(rows, v, device="cuda").normal_(std=3.0, generator=gen)
    raised = torch.randint(0, v, (rows, 8), device="cuda", generator=gen)
    logits.scatter_add_(1, raised, 6.0 * torch.rand(rows, 8, device="cuda", generator=gen))
    scores = torch.empty(g, b, device="cuda").normal_(mean=0.0, std=1.5, generator=gen) - 20.0
    ended = torch.rand(g, b, device="cuda", generator=gen) * 100 < case["ended"]
    ended[:, 0] = False
    if case["first"]:
        scores[:, 0], scores[:, 1:], ended[:] = 0.0, -math.inf, False
    carried = []
    if case["history"]:
        carried.append(torch.randint(0, v, (rows, case["history"]), dtype=torch.int32, device="cuda", generator=gen))
    carried += [_normal(gen, (rows, case["state"]), torch.float16) for _ in range(case["layers"])]
    return {"case": case, "logits": logits.to(_dtype(case)), "scores": scores.view(-1), "ended": ended.view(-1), "carried": carried,
            "next": [torch.empty_like(t) for t in carried]}


def prepare(case, seed):
    if case["kind"] == "beam":
        return _beam_state(case, seed)
    state = _cache_state(case, seed)
    if own:
        import paper_2503_23294_amd as ck
        # handles on the same tensors, as a program keeps them
        state["pages"] = ck.PageTable.of(state["table"], state["lens"], state["refs"], case["page"])
        state["cache"] = ck.Kv16Cache(state["pages"], case["kv_heads"], case["head_dim"], _dtype(case), pools=(state["pool_k"], state["pool_v"]))
        if case["kind"] == "append":
            state["rotation"] = ck.Rotation(state["inv_freq"], interleaved=case["interleaved"])
    return state


# ---- the plain form ------------------------------------------------------------------------------------------------------


def _rows(starts, lens, total):
    """Sequence, position in the sequence and number among the new tokens of each of `total` new tokens."""
    t = torch.arange(total, device=starts.device)
    row = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    i = t - starts[row]
    return row, lens[row].long() - (starts[row + 1] - starts[row]) + i, i


def _rotate(case, x, cos, sin):
    """x: [tokens, heads, D]; cos, sin: [tokens, 1, rotary / 2]."""
    r = case["rotary"]
    y = x.float()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if case["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=-1).flatten(-2) if case["interleaved"] else torch.cat([a, b], dim=-1)
    return torch.cat([turned, y[..., r:]], dim=-1).to(x.dtype)


def _plain_append(state):
    case, p = state["case"], state["case"]["page"]
    row, pos, _ = _rows(state["starts"], state["lens"], state["k"].shape[0])
    angle = (pos[:, None].double() * state["inv_freq"])[:, None]           # far positions: 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    page, at = state["table"][row, pos // p].long(), pos % p
    state["pool_k"][page, :, at] = _rotate(case, state["k"], cos, sin)
    state["pool_v"][page, :, at] = state["v"]
    return {"k": state["pool_k"], "v": state["pool_v"], "q": _rotate(case, state["q"], cos, sin)}


def _plain_attend(state):
    case, q, lens, starts = state["case"], state["q"], state["lens"], state["starts"]
    h, d, p = case["kv_heads"], case["head_dim"], case["page"]
    rep, total, n, batch = case["q_heads"] // h, q.shape[0], case["new"], case["batch"]
    cols = -(-case["tokens"] // p)
    pages = state["table"][:, :cols].clamp(min=0).long()
    tokens = torch.arange(cols * p, device=q.device)
    there = (tokens < lens[:, None])[:, None, :, None]
    # [B, heads, T, D]
    k = torch.where(there, state["pool_k"][pages].transpose(1, 2).flatten(2, 3).float(), 0.0)
    v = torch.where(there, state["pool_v"][pages].transpose(1, 2).flatten(2, 3).float(), 0.0)
    row, pos, i = _rows(starts, lens, total)
    padded = torch.zeros(batch, n, h, rep, d, device=q.device)
    padded[row, i] = q.float().view(total, h, rep, d)
    last = torch.full((batch, n), -1, dtype=torch.int64, device=q.device)
    last[row, i] = pos
    # [B, heads, rep, n, D] x [B, heads, D, T]
    s = torch.matmul(padded.permute(0, 2, 3, 1, 4).reshape(batch, h, rep * n, d), k.transpose(2, 3).contiguous())
    s = s.view(batch, h, rep, n, -1) * (1 / math.sqrt(d))
    s.masked_fill_((tokens > last[..., None])[:, None, None], -math.inf)
    top = s.amax(dim=-1, keepdim=True).clamp(min=-1e30)
    weight = torch.exp(s.sub_(top))
    total_weight = weight.sum(dim=-1, keepdim=True)
    o = torch.matmul(weight.view(batch, h, rep * n, -1), v).view(batch, h, rep, n, d)
    o = o / torch.where(total_weight > 0, total_weight, 1.0)
    lse = top + torch.log(total_weight)
    return {"out": o.permute(0, 3, 1, 2, 4)[row, i].flatten(1, 2).to(q.dtype), "lse": lse[..., 0].permute(0, 3, 1, 2)[row, i].flatten(1, 2)}


def _plain_beam(state):
    case, x = state["case"], state["logits"]
    g, b, v, keep = case["groups"], case["beams"], case["vocab"], case["keep"]
    x = x.double()                                                         # values next to the border of what is kept
    top = x.amax(dim=1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(dim=1, keepdim=True))
    before = state["scores"].double()[:, None]
    total = before + (x - lse)
    only_eos = torch.full_like(total, -math.inf)
    only_eos[:, EOS] = before[:, 0]
    total = torch.where(state["ended"][:, None], only_eos, total).view(g, b * v)
    score, place = torch.sort(total, dim=1, descending=True, stable=True)  # ties go to the lowest index
    score, place = score[:, :keep], place[:, :keep]
    there = score > -math.inf
    source = torch.where(there, place // v + b * torch.arange(g, device=x.device)[:, None], -1)
    token = torch.where(there, place % v, -1)
    ended = state["ended"][source.clamp(min=0)] & there | (token == EOS)
    for to, of in zip(state["next"], state["carried"]):
        to.copy_(torch.where((source >= 0).view(-1, 1), of[source.clamp(min=0).view(-1)], to))
    return {"source": source.int(), "token": token.int(), "score": score.float(), "ended": ended, "carried": state["next"]}


# ---- the pass --------------------------------------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "beam": _plain_beam}[case["kind"]](state)
    import paper_2503_23294_amd as ck
    if case["kind"] == "append":
        q = ck.cocktail_kv16_append(state["cache"], state["k"], state["v"], state["starts"], state["rotation"], q=state["q"])
        return {"k": state["pool_k"], "v": state["pool_v"], "q": q}
    if case["kind"] == "attend":
        out, lse = ck.cocktail_kv16_attention(state["cache"], state["q"], state["starts"], max_new=case["new"], max_len=case["tokens"])
        return {"out": out, "lse": lse}
    source, token, score, ended = ck.cocktail_beam_select(state["logits"], state["scores"], case["beams"], keep=case["keep"], eos=EOS,
                                                          finished=state["ended"])
    if state["carried"]:
        ck.cocktail_beam_reorder(source, state["carried"], out=state["next"])
    return {"source": source, "token": token, "score": score, "ended": ended, "carried": state["next"]}


def work(case):
    if case["kind"] == "beam":
        rows = case["groups"] * case["beams"]
        values = rows * case["vocab"]
        carried = rows * (4 * case["history"] + 2 * case["state"] * case["layers"])
        return {"bytes": values * (4 if case["dtype"] == "float32" else 2) + 2 * carried + 5 * rows + 13 * case["groups"] * case["keep"],
                "flops": 4 * values}
    d, h, hq = case["head_dim"], case["kv_heads"], case["q_heads"]
    lens, new = _lengths(case)
    if case["kind"] == "append":
        return {"bytes": sum(new) * (2 * h + hq) * d * 4, "flops": 3 * sum(new) * (h + hq) * case["rotary"]}
    pairs = sum(n * t - n * (n - 1) // 2 for t, n in zip(lens, new))
    return {"bytes": sum(lens) * h * d * 4 + sum(new) * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}


# ---- the definition, apart from the above ------------------------------------------------------------------------------------


def _turned(x, pos, case):
    """x [tokens, heads, D] in 64 bits, every pair of channels as a complex number times e^(i * angle)."""
    r, pairs = case["rotary"], case["rotary"] // 2
    y = x.double().clone()
    step = torch.tensor([case["base"] ** (-2.0 * i / r) for i in range(pairs)], dtype=torch.float64, device=x.device)
    turn = torch.polar(torch.ones(len(pos), pairs, dtype=torch.float64, device=x.device), pos.double()[:, None] * step)[:, None]
    index = torch.arange(pairs, device=x.device)
    re, im = (2 * index, 2 * index + 1) if case["interleaved"] else (index, index + pairs)
    z = torch.complex(y[..., re], y[..., im]) * turn
    y[..., re], y[..., im] = z.real, z.imag
    return y


def _exact_append(case, seed):
    state = _cache_state(case, seed)
    lens, new = _lengths(case)
    k, v = state["pool_k"].double(), state["pool_v"].double()
    q = torch.empty(state["q"].shape, dtype=torch.float64, device="cuda")
    first, p = 0, case["page"]
    for b, (t, n) in enumerate(zip(lens, new)):
        pos = torch.arange(t - n, t, device="cuda")
        rows = slice(first, first + n)
        q[rows] = _turned(state["q"][rows], pos, case)
        keys, values = _turned(state["k"][rows], pos, case), state["v"][rows].double()
        pages = state["table"][b].tolist()
        for col in range((t - n) // p, (t - 1) // p + 1):
            lo, hi, page = max(t - n, col * p), min(t, (col + 1) * p), pages[col]
            k[page, :, lo - col * p:hi - col * p] = keys[lo - t + n:hi - t + n].transpose(0, 1)
            v[page, :, lo - col * p:hi - col * p] = values[lo - t + n:hi - t + n].transpose(0, 1)
        first += n
    return {"k": k, "v": v, "q": q}


def _exact_attend(case, seed):
    lens, new = _lengths(case)
    d, h, p = case["head_dim"], case["kv_heads"], case["page"]
    rep = case["q_heads"] // h
    if 8 * d * case["q_heads"] * sum(n * t for t, n in zip(lens, new)) > 2e13:
        return None
    state = _cache_state(case, seed)
    q = state["q"]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
    first = 0
    for b, (t, n) in enumerate(zip(lens, new)):
        pages = state["table"][b, :-(-t // p)].long()
        seen = torch.arange(t, device="cuda") <= torch.arange(t - n, t, device="cuda")[:, None]
        for i in range(h):
            ks, vs = (state[x][pages, i].flatten(0, 1)[:t].double() for x in ("pool_k", "pool_v"))
            for j in range(i * rep, (i + 1) * rep):
                s = torch.where(seen, q[first:first + n, j].double() @ ks.t() / math.sqrt(d), -math.inf)
                lse[first:first + n, j] = torch.logsumexp(s, dim=1)
                out[first:first + n, j] = torch.softmax(s, dim=1) @ vs
        first += n
    return {"out": out, "lse": lse}


def _exact_beam(case, seed):
    state = _beam_state(case, seed)
    g, b, v, keep = case["groups"], case["beams"], case["vocab"], case["keep"]
    scores, ended = state["scores"].tolist(), state["ended"].tolist()
    # no row has more than `keep` of the best; among equals of a row the first ones are wanted: those from the value on that `keep` reach
    x = state["logits"].double()
    lse = torch.logsumexp(x, dim=1).tolist()
    border = torch.topk(x, min(keep, v), dim=1).values[:, -1:]
    rows, cols = torch.nonzero(x >= border, as_tuple=True)
    found = [[] for _ in range(g * b)]
    for r, c, y in zip(rows.tolist(), cols.tolist(), x[rows, cols].tolist()):
        found[r].append((c, y))
    source, token, score, over = [], [], [], []
    for i in range(g):
        candidates = []
        for r in range(i * b, (i + 1) * b):
            if ended[r]:
                candidates.append((-scores[r], r, EOS))
            else:
                candidates += [(-(scores[r] + (y - lse[r])), r, c) for c, y in found[r]]
        best = sorted(c for c in candidates if c[0] < math.inf)[:keep]
        best += [(math.inf, -1, -1)] * (keep - len(best))
        source.append([r for _, r, _ in best])
        token.append([c for _, _, c in best])
        score.append([-s for s, _, _ in best])
        over.append([r >= 0 and (ended[r] or c == EOS) for _, r, c in best])
    source = torch.tensor(source, dtype=torch.int32, device="cuda")
    carried = []
    for t in state["carried"]:
        carried.append(torch.stack([t[r] for r in source.view(-1).tolist()]))
    return {"source": source, "token": torch.tensor(token, dtype=torch.int32, device="cuda"),
            "score": torch.tensor(score, dtype=torch.float64, device="cuda"), "ended": torch.tensor(over, device="cuda"), "carried": carried}


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend, "beam": _exact_beam}[case["kind"]](case, seed)
