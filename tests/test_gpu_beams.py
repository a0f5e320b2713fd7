"""The beam search's selection against its definition in float64: ties, ended candidates, masked and broken rows.

Scores are rounded to fp32 once (2^-24) from fp32 sums of exponentials of at most 4096 values a part (2^-24 each,
and the exponential's error of some 2^-22): 1e-6 of the log sum; integers are equal."""
import numpy as np
import pytest
import torch

import synth
from paper_2607_01125_amd import generate as G
from paper_2607_01125_amd import zoact as Z

import packed_ref as ref
from gpu_helpers import announce, dev, host, t_bf16, t_f32, t_i32
from test_gpu_generate import _prompts, _tuned

pytestmark = pytest.mark.gpu


def _select(logits, score, hist, length, eos, kept, bf16=False, pad=0):
    n, bi = score.shape
    V = logits.shape[1]
    wide = np.full((n * bi, V + pad), 1.0e30, np.float32)
    wide[:, :V] = logits
    lg = (t_bf16(wide) if bf16 else t_f32(wide))[:, :V]
    to = Z.Beams(torch.full((n, kept), -7.0, device=dev()),
                 torch.full((n, kept, length + 3), -7, dtype=torch.int32, device=dev()))
    tok, src = (torch.full((n * kept,), -7, dtype=torch.int32, device=dev()) for _ in range(2))
    ws = torch.full((Z.beam_workspace_bytes(n, bi, kept, V),), 255, dtype=torch.uint8, device=dev())
    Z.beam_select(lg, Z.Beams(t_f32(score), t_i32(hist)), length, eos, to, tok, src, ws)
    return to, tok, src


def _check(logits, score, hist, length, eos, kept, **kw):
    to, tok, src = _select(logits, score, hist, length, eos, kept, **kw)
    n, bi = score.shape
    got, gh = host(to.score), to.hist.cpu().numpy()
    tok, src = tok.cpu().numpy().reshape(n, kept), src.cpu().numpy().reshape(n, kept)
    for i in range(n):
        val, beam, token = ref.beams(logits[i * bi:(i + 1) * bi].astype(np.float64), score[i], hist[i], length,
                                     -1 if eos is None else eos, kept)
        assert np.array_equal(tok[i], token) and np.array_equal(src[i], i * kept + beam), (i, tok[i], token, src[i], beam)
        assert np.array_equal(gh[i, :, :length], hist[i][beam, :length]) and np.array_equal(gh[i, :, length], token)
        assert (gh[i, :, length + 1:] == -7).all()
        same = np.array_equal(np.isnan(got[i]), np.isnan(val)) and np.array_equal(np.isinf(got[i]), np.isinf(val))
        assert same, (i, got[i], val)
        f = np.isfinite(val)
        assert np.all(np.abs(got[i][f] - val[f]) <= 2.0 ** -24 * np.abs(val[f]) + 2e-5)


def _case(n, bi, V, length, seed, bf16=False):
    lg = synth.normal((n * bi, V), 2.5, seed, V, bi)
    lg = synth.bf16_round(lg) if bf16 else lg
    score = (-synth.gen(seed, 5).random((n, bi)) * 4 - length).astype(np.float32)
    hist = synth.gen(seed, 6).integers(3, max(V, 4), (n, bi, length + 2)).astype(np.int32)
    return lg, score, hist


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,bi,kept,V,length", [
    (1, 1, 1, 1, 0), (2, 1, 4, 7, 0), (3, 4, 4, 512, 5), (2, 3, 5, 4097, 1), (5, 2, 2, 8191, 40), (1, 16, 16, 50272, 17),
    (2, 64, 64, 300, 3), (1, 7, 64, 12289, 2), (1, 64, 64, 64, 9), (3, 1, 64, 4160, 0), (40, 5, 5, 1001, 3)])
def test_against_the_definition(n, bi, kept, V, length, bf16):
    announce("beam_select", n, bi, kept, V, length, bf16)
    lg, score, hist = _case(n, bi, V, length, 1, bf16)
    _check(lg, score, hist, length, 2 if V > 2 else None, kept, bf16=bf16)
    _check(lg, score, hist, length, None, kept, bf16=bf16, pad=4)
    _check(lg, score, hist, length, None, kept, bf16=bf16, pad=3)


def test_ended_candidates_stay_and_compete():
    lg, score, hist = _case(4, 4, 600, 6, 2)
    score[:] = -20.0 - np.arange(16).reshape(4, 4) * 0.5
    hist[0, :, 5] = 9                              # all of a prompt
    hist[1, 0, 5] = hist[2, 3, 5] = hist[2, 1, 5] = 9
    hist[3, :, 4] = 9                              # an earlier token: not ended
    announce("beam_select ended")
    _check(lg, score, hist, 6, 9, 4)
    _check(lg, score, hist, 6, 9, 2)
    _check(lg, score, hist, 6, 9, 7)               # more than are alive: -inf from the lowest beam on
    _check(lg, score, hist, 6, None, 4)
    hist[:, :, 5] = 0
    _check(lg, score, hist, 6, 0, 4)
    _check(lg, score, hist, 0, 0, 4)               # (no token yet: nobody has ended)


@pytest.mark.parametrize("V", [90, 5000, 20000])
@pytest.mark.parametrize("kept", [1, 4, 33, 64])
def test_equal_logits_and_masked_vocabularies(kept, V):
    """Ties go to the lowest beam and token, also where very many are equal; -inf is taken last."""
    announce("beam_select ties", kept, V)
    lg, score, hist = _case(3, 2, V, 2, 3)
    _check(np.zeros_like(lg), np.zeros_like(score), hist, 2, None, kept)
    _check(np.round(lg), np.zeros_like(score), hist, 2, None, kept)
    masked = lg.copy()
    masked[:, synth.gen(3, 9).permutation(V)[3:]] = -np.inf          # three tokens left
    _check(masked, score, hist, 2, None, kept)
    masked = lg.copy()
    masked[:, :V - V // 8] = -np.inf
    _check(masked, score, hist, 2, None, kept)
    # zeros of either sign are equal
    z = np.full_like(lg, -5.0)
    z[:, 11::7] = 0.0
    z[:, 4::7] = -0.0
    _check(z, np.zeros_like(score), hist, 2, None, kept)


def test_rows_that_are_not_numbers():
    """A NaN or +inf among a row's logits, nothing but -inf, and scores that are no sums of log probabilities."""
    lg, score, hist = _case(7, 3, 9000, 2, 4)
    lg[1, 8000] = np.nan
    lg[3 + 2, 17] = np.inf
    lg[6 + 0] = -np.inf
    lg[9 + 1, :] = np.nan
    score[4, 1], score[4, 2] = -np.inf, -np.inf
    score[5, 0] = np.nan
    score[6, 1] = np.inf
    hist[4, 2, 1] = 5
    announce("beam_select not numbers")
    for kept in (1, 3, 40):
        _check(lg, score, hist, 2, 5, kept)
    score[4, 0] = -np.inf
    _check(lg, score, hist, 2, 5, 3)


def test_large_and_small_logits():
    """Differences from the log sum far below one step of the logits, and rows 1e4 apart."""
    lg, score, hist = _case(2, 3, 3000, 2, 5)
    lg *= 1.0e-3
    lg[1::2] += 1.0e4
    announce("beam_select far")
    to, tok, src = _select(lg, score, hist, 2, None, 3)
    for i in range(2):
        val, beam, token = ref.beams(lg[i * 3:i * 3 + 3].astype(np.float64), score[i], hist[i], 2, -1, 3)
        assert np.array_equal(tok.cpu().numpy()[i * 3:i * 3 + 3], token)
        assert np.abs(host(to.score)[i] - val).max() < 1e-4


def test_lists_that_are_not_wanted_and_a_graph():
    lg, score, hist = _case(2, 4, 700, 3, 6)
    t, now = t_f32(lg), Z.Beams(t_f32(score), t_i32(hist))
    to = Z.Beams.alloc(2, 4, 5, dev())
    tok, src = (torch.zeros(8, dtype=torch.int32, device=dev()) for _ in range(2))
    ws = torch.empty(Z.beam_workspace_bytes(2, 4, 4, 700), dtype=torch.uint8, device=dev())
    announce("beam_select graph")
    Z.beam_select(t, now, 3, 2, to, None, None, ws)
    first = to.score.clone(), to.hist.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        Z.beam_select(t, now, 3, 2, to, tok, src, ws)
    for seed in (6, 7, 8):
        lg, score, hist = _case(2, 4, 700, 3, seed)
        t.copy_(t_f32(lg))
        now.score.copy_(t_f32(score))
        now.hist.copy_(t_i32(hist))
        for x in (to.score, to.hist, tok, src):
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        if seed == 6:
            assert torch.equal(to.score, first[0]) and torch.equal(to.hist[:, :, :4], first[1][:, :, :4])
        for i in range(2):
            _, beam, token = ref.beams(lg[i * 4:i * 4 + 4].astype(np.float64), score[i], hist[i], 3, 2, 4)
            assert np.array_equal(tok.cpu().numpy()[i * 4:i * 4 + 4], token)
            assert np.array_equal(src.cpu().numpy()[i * 4:i * 4 + 4], i * 4 + beam)


def test_more_beams_than_the_kernel_keeps():
    """65 beams take the plain way: the best of 64 and of 65 agree where they share the first."""
    shape = synth.shrink(synth.TINY, vocab=128)
    _, g, _ = _tuned(shape, "fp32")
    prompts = _prompts(shape, [9], 23)
    announce("many beams")
    assert g.generate(prompts, 2, beams=65) == g.generate(prompts, 2, beams=64)
    assert g.generate(prompts, 1, beams=65) == g.generate(prompts, 1)


def test_the_selection_and_the_torch_way_choose_alike():
    lg, score, hist = _case(3, 5, 900, 4, 9)
    hist[1, 2, 3] = 7
    to, tok, src = _select(lg, score, hist, 4, 7, 5)
    other = Z.Beams.alloc(3, 5, 7, dev())
    t2, s2 = torch.empty_like(tok), torch.empty_like(src)
    G._select_many(t_f32(lg), Z.Beams(t_f32(score), t_i32(hist)), 4, 7, other, t2, s2, None)
    assert torch.equal(tok, t2) and torch.equal(src, s2) and torch.equal(to.hist[:, :, :5], other.hist[:, :, :5])
    assert float((to.score - other.score).abs().max()) < 1e-4


def test_rows_of_logits_further_apart_than_32_bits():
    far = 2 ** 31 + 64
    buf = torch.zeros(far + 4096, device=dev())
    lg, score, hist = _case(2, 1, 600, 3, 17)
    wide = buf.as_strided((2, 600), (far, 1))
    wide.copy_(t_f32(lg))
    announce("beam_select rows far apart")
    want, tok, src = _select(lg, score, hist, 3, None, 5)
    to, t2, s2 = Z.Beams.alloc(2, 5, want.hist.shape[2], dev()), torch.empty_like(tok), torch.empty_like(src)
    ws = torch.empty(Z.beam_workspace_bytes(2, 1, 5, 600), dtype=torch.uint8, device=dev())
    Z.beam_select(wide, Z.Beams(t_f32(score), t_i32(hist)), 3, None, to, t2, s2, ws)
    assert torch.equal(t2, tok) and torch.equal(s2, src) and torch.equal(to.score, want.score)
