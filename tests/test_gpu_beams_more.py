"""The beam search's selection where candidates are most: more than a workgroup reads at once, more equal ones than it
ranks at once, rows of more parts than a wave has lanes.  Tolerances as in test_gpu_beams."""
import numpy as np
import pytest

import synth

from gpu_helpers import announce
from test_gpu_beams import _case, _check, _select

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [300, 5000])
def test_rows_that_are_not_numbers_of_very_many_beams(V):
    """64 beams whose rows all hold a NaN: every candidate is NaN, and the lowest 64 (beam, token) are kept; then all
    but a few such rows, in which the first beam is among them and is not."""
    lg, score, hist = _case(1, 64, V, 3, 21)
    broken = lg.copy()
    broken[:, V // 2] = np.nan
    announce("beam_select all NaN", V)
    _check(broken, score, hist, 3, None, 64)
    _check(broken, score, hist, 3, None, 1)
    broken[5:9] = lg[5:9]
    _check(broken, score, hist, 3, None, 64)
    broken[0] = lg[0]
    _check(broken, score, hist, 3, None, 64)
    _check(broken, score, hist, 3, None, 7)


@pytest.mark.parametrize("kept", [1, 33, 64])
@pytest.mark.parametrize("V", [300, 5000, 8193])
def test_more_candidates_than_are_read_at_once(V, kept):
    """64 beams of one to three parts: up to 12288 candidates, drawn, all alike, of few values, and of lost beams."""
    lg, score, hist = _case(2, 64, V, 4, 22)
    announce("beam_select many candidates", V, kept)
    _check(lg, score, hist, 4, 2, kept)
    _check(np.zeros_like(lg), np.zeros_like(score), hist, 4, None, kept)
    _check(np.round(lg), np.zeros_like(score), hist, 4, None, kept)
    lost = np.full_like(score, -np.inf)
    _check(lg, lost, hist, 4, None, kept)
    lost[0, 40], lost[1, 63] = -2.0, -5.0
    _check(lg, lost, hist, 4, None, kept)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,bi,kept,V", [(1, 1, 5, 262144 + 3 * 4096 + 5), (1, 2, 64, 300000), (2, 1, 4, 262144 + 4096)])
def test_rows_of_more_parts_than_a_wave_has_lanes(n, bi, kept, V, bf16):
    lg, score, hist = _case(n, bi, V, 2, 23, bf16)
    announce("beam_select many parts", n, bi, kept, V, bf16)
    _check(lg, score, hist, 2, None, kept, bf16=bf16)
    lg[:, synth.gen(23, 1).permutation(V)[: V - V // 7]] = -np.inf
    _check(lg, score, hist, 2, None, kept, bf16=bf16, pad=3)


@pytest.mark.parametrize("bi,V,kept", [(2, 300, 9), (2, 6000, 9), (2, 6000, 1), (1, 300, 4), (64, 300, 64)])
def test_logits_closer_than_their_values_resolve(bi, V, kept):
    """Logits of 1e-20 and their like beside a log sum of some units: equal values in 64 bits.  Within a beam the larger
    logit comes first, then the lower token; between beams the larger value, then the lower beam."""
    lg = np.full((bi, V), -5.0, np.float32)
    rng = synth.gen(24, V, bi)
    at = np.r_[V - 7, rng.permutation(V - 7)[:39]]          # (the same of every beam, so that the log sums are equal)
    lg[:, at] = np.float32(1.0e-20) * rng.integers(-3, 4, (bi, 40)).astype(np.float32)
    lg[0, V - 7] = np.float32(9.0e-20)
    score, hist = np.zeros((1, bi), np.float32), np.zeros((1, bi, 3), np.int32)
    x = lg.astype(np.float64)
    lse = x.max(axis=1) + np.log(np.exp(x - x.max(axis=1)[:, None]).sum(axis=1))
    assert np.unique((x - lse[:, None])[x > -1.0]).size == 1
    order = sorted((-(x[j, v] - lse[j]), j, -x[j, v], v) for j in range(bi) for v in range(V))[:kept]
    announce("beam_select unresolved logits", bi, V, kept)
    to, tok, src = _select(lg, score, hist, 1, None, kept)
    assert src.tolist() == [o[1] for o in order] and tok.tolist() == [o[3] for o in order]


@pytest.mark.parametrize("bi,kept,V", [(16, 16, 50272), (33, 33, 9000), (48, 48, 9000), (49, 49, 9000), (64, 64, 20000)])
def test_long_histories_whose_scores_are_near_one_another(bi, kept, V):
    """Scores of about -1500 within a few of each other, which differ in the lower bits of their order only."""
    lg, score, hist = _case(2, bi, V, 5, 25)
    score[0] = -1500.0 - 2.0 * synth.gen(25, 3).random(bi).astype(np.float32)
    score[1] = -90.0 - 40.0 * synth.gen(25, 4).random(bi).astype(np.float32)
    announce("beam_select long histories", bi, kept, V)
    _check(lg, score, hist, 5, 2, kept)
