"""The order of beam search's selection: ties between rows, and what does not depend on where in memory the logits lie."""
import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck
from oracle import kv16_oracle as O

gpu = pytest.mark.gpu
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("vocab", [1, 7, 509, 1001, 4099, 50257, 65001])
def test_equal_rows_at_equal_scores_are_in_the_order_of_their_rows(vocab, dtype):
    """Rows that are alike have the same sum of exponentials to the last bit, wherever each of them begins: a logit's continuations come out row by row."""
    rng = np.random.default_rng(vocab)
    for beams, keep in ((2, 6), (4, 8), (8, 5), (64, 64)):
        row = torch.from_numpy(rng.standard_normal(vocab) * 3).to("cuda:0", DTYPES[dtype])
        got = ck.cocktail_beam_select(row.repeat(2 * beams, 1), torch.full((2 * beams,), -1.25, device="cuda:0"), beams, keep=keep)
        # the largest logits, the lower token first; every one of them in every row
        best = np.lexsort((np.arange(vocab), -row.double().cpu().numpy()))
        value = row.double().cpu().numpy()[best]
        order = sorted(((-x, r, int(v)) for x, v in zip(value[:keep], best[:keep]) for r in range(beams)))[:keep]
        for g in range(2):
            n = min(keep, vocab * beams)
            assert got[0][g, :n].tolist() == [r + g * beams for _, r, _ in order], (beams, keep)
            assert got[1][g, :n].tolist() == [v for _, _, v in order], (beams, keep)
            assert (got[0][g, n:] == -1).all()
        assert torch.equal(got[2][0], got[2][1])


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("vocab", [777, 4001, 50257])
def test_a_view_selects_as_a_copy_does(vocab, dtype):
    """The same rows at every address that their elements may have: the same results, scores bit by bit."""
    rng = np.random.default_rng(vocab + 1)
    logits = torch.from_numpy(rng.standard_normal((6, vocab)) * 3).to("cuda:0", DTYPES[dtype])
    logits[3:] = logits[:3]
    scores = torch.tensor([-1.0, -2.0, -1.5] * 2, device="cuda:0")
    want = ck.cocktail_beam_select(logits, scores, 6, keep=24)
    for offset in range(17):
        wide = torch.full((6, vocab + 29), 1e4, dtype=logits.dtype, device="cuda:0")
        view = wide[:, offset:offset + vocab]
        view.copy_(logits)
        got = ck.cocktail_beam_select(view, scores, 6, keep=24)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), offset
    # rows that begin at other places of a line each
    flat = torch.full((6 * (vocab + 5),), 1e4, dtype=logits.dtype, device="cuda:0")
    view = flat.as_strided((6, vocab), (vocab + 5, 1), 3)
    view.copy_(logits)
    assert all(torch.equal(x, y) for x, y in zip(ck.cocktail_beam_select(view, scores, 6, keep=24), want))


# ---- every place of a selection -------------------------------------------------------------------------------------------------------

# What a candidate's value may be off by, in binary64.  Terms of a sum of exponentials are 2^((x - ref) log2(e)): the difference, the constant and the product
# are rounded, 2.5 * 2^-24 |x - ref| of the term, the function and sums of eight in binary32 are another 9 * 2^-24.  A reference is 16 below the largest logit at
# most, and the distance to that one is ln(vocab) <= 17 at most in the mean over the terms, by their weights: 92 * 2^-24.  Sums of waves, pieces and rows are
# brought to one reference, up to three times, with factors of 16 at most where they count: 42 * 2^-24 each.
VALUE = 2.0 ** -16


def check_places(logits, scores, beams, keep, eos, finished, got):
    """Raises where the selection is not the right one.  Continuations of one row have its sum in common: they are the first ones of the row, in their order, to
    the last bit.  Those of different rows may only be exchanged where their values are as near as what they may be off by."""
    source, token, score, over = (np.asarray(x) for x in got)
    x = np.asarray(logits, np.float64)
    for g in range(len(x) // beams):
        orders, values = {}, {}
        wanted = []
        for r in range(g * beams, (g + 1) * beams):
            if not scores[r] > -np.inf:
                orders[r], values[r] = [], {}
            elif finished is not None and finished[r]:
                orders[r], values[r] = [eos], {eos: float(scores[r])}
            else:
                logp = O.log_probabilities(x[r])
                clean = np.where(logp > -np.inf, np.minimum(x[r], float(np.finfo(np.float32).max)), -np.inf)
                best = np.lexsort((np.arange(len(clean)), -clean))[:keep + 1]
                orders[r] = [int(v) for v in best if logp[v] > -np.inf]
                values[r] = {v: float(scores[r]) + logp[v] for v in orders[r]}
            wanted += [(-values[r][v], r, i, v) for i, v in enumerate(orders[r])]
        wanted.sort()
        there = min(keep, len(wanted))
        assert (source[g, there:] == -1).all() and (token[g, there:] == -1).all() and np.isneginf(score[g, there:]).all() and not over[g, there:].any(), g
        taken = {r: 0 for r in orders}
        for i in range(there):
            r, v = int(source[g, i]), int(token[g, i])
            assert r in orders and taken[r] < len(orders[r]) and orders[r][taken[r]] == v, (g, i, r, v)
            taken[r] += 1
            own, want = values[r][v], -wanted[i][0]
            assert abs(float(score[g, i]) - own) <= VALUE + 2.0 ** -24 * abs(own), (g, i, float(score[g, i]), own)
            assert abs(own - want) <= 2 * VALUE, (g, i, own, want)
            others = [-wanted[k][0] for k in (i - 1, i + 1) if 0 <= k < len(wanted)]
            if all(abs(want - o) > 2 * VALUE for o in others):
                assert (r, v) == (wanted[i][1], wanted[i][3]), (g, i, r, v, wanted[i])
            assert bool(over[g, i]) == (v == eos or bool(finished is not None and finished[r])), (g, i)


def _problem(rng, groups, beams, vocab, dtype, ended):
    rows = groups * beams
    logits = torch.from_numpy(rng.standard_normal((rows, vocab)) * 3).to(dtype)
    scores = rng.standard_normal(rows).astype(np.float32) - 20
    return logits, scores, (rng.random(rows) < 0.3) if ended else None


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("groups,beams,vocab,keep,ended", [(2, 1, 3000, 1, False), (2, 4, 500, 4, True), (1, 5, 2000, 3, False), (3, 2, 300, 64, True), (1, 8, 40000, 8, True)])
def test_a_wrong_place_is_seen(groups, beams, vocab, keep, ended, dtype):
    """The oracle's own selection passes; one mistake anywhere in it does not, the last place included."""
    rng = np.random.default_rng(vocab + keep)
    logits, scores, finished = _problem(rng, groups, beams, vocab, DTYPES[dtype], ended)
    x, eos = logits.double().numpy(), 7
    right = O.select(x, scores.tolist(), beams, keep, eos, finished)
    right = (right[0], right[1], right[2].astype(np.float32), right[3])
    args = (x, scores, beams, keep, eos, finished)
    check_places(*args, right)

    def wrong(change):
        got = [np.array(a) for a in right]
        change(*got)
        with pytest.raises(AssertionError):
            check_places(*args, got)
    for g in range(groups):
        for i in range(keep):
            def another_token(source, token, score, over):
                token[g, i] = (token[g, i] + 1234) % vocab

            def next_token(source, token, score, over):
                token[g, i] = (token[g, i] + 1) % vocab

            def another_row(source, token, score, over):
                source[g, i] = g * beams + (source[g, i] + 1) % beams if beams > 1 else source[g, i] + 1

            def another_score(source, token, score, over):
                score[g, i] += 1e-3

            def another_end(source, token, score, over):
                over[g, i] = not over[g, i]

            def none(source, token, score, over):
                source[g, i] = token[g, i] = -1

            def twice(source, token, score, over):
                k = (i + 1) % keep
                source[g, i], token[g, i], score[g, i], over[g, i] = source[g, k], token[g, k], score[g, k], over[g, k]
            for change in (another_token, next_token, another_row, another_score, another_end, none) + ((twice,) if keep > 1 else ()):
                wrong(change)
        # the best one is missing, the others move up, and the first that is left out takes the last place
        more = O.select(x, scores.tolist(), beams, min(64, keep + 1), eos, finished)

        def moved(source, token, score, over):
            for a, b in zip((source, token, score, over), more):
                a[g, :min(keep, b.shape[1] - 1)] = b[g, 1:keep + 1]
        if keep < 64:
            wrong(moved)


@gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("groups,beams,vocab,keep", [(1, 1, 1, 1), (1, 4, 1, 4), (2, 3, 7, 5), (1, 4, 32000, 4), (3, 8, 5003, 8), (2, 64, 999, 64), (5, 5, 4096, 10),
                                                     (1, 64, 20011, 64), (40, 2, 513, 2), (300, 4, 2049, 4), (2, 1, 300001, 64), (1, 16, 8191, 32), (9, 1, 50257, 1), (64, 8, 2047, 8)])
def test_every_place(groups, beams, vocab, keep, dtype):
    rng = np.random.default_rng(vocab * 3 + keep)
    eos = vocab // 2
    for ended in (False, True):
        logits, scores, finished = _problem(rng, groups, beams, vocab, DTYPES[dtype], ended)
        got = ck.cocktail_beam_select(logits.cuda(), torch.from_numpy(scores).cuda(), beams, keep=keep, eos=eos,
                                      finished=None if finished is None else torch.from_numpy(finished).cuda())
        check_places(logits.double().numpy(), scores, beams, keep, eos, finished, [t.cpu().numpy() for t in got])
