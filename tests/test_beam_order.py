"""The order of beam search's selection: ties between rows, and what does not depend on where in memory the logits lie."""
import numpy as np
import pytest
import torch

import paper_2503_23294_amd as ck

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
