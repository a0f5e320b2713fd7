"""The cache, its attention, the matrix-vector products and the pages as a model uses them: sessions over
whole decoders against the oracle's forward with keys and values quantised as the cache holds them."""
import math

import numpy as np
import pytest
import torch

import synth
from oracle import model as om
from paper_2607_01125_amd import generate as G
from paper_2607_01125_amd import zoact as Z

from gpu_helpers import announce, dev, host
from test_gpu_model import LLAMA_S, OPT_S, _logits_close, _models

pytestmark = pytest.mark.gpu

MODELS = [(synth.TINY, "fp32"), (LLAMA_S, "bf16"), (LLAMA_S, "int4"), (OPT_S, "bf16"), (OPT_S, "int4")]
IDS = ["tiny-fp32", "llama-bf16", "llama-int4", "opt-bf16", "opt-int4"]


def _tuned(shape, mode, seed=3):
    """Oracle and GPU model with coefficients as after some training."""
    o, g = _models(shape, mode, seed, perturb=True)
    c = synth.normal((o.k,), 0.05, seed, 77)
    c = synth.bf16_round(c) if g.c_bf16 else c
    g.arena.c.copy_(torch.from_numpy(c))
    return o, g, c


def _as_cached(x):
    """Blocks of 16 tokens of a head as codes and one scale, and back; x float64 [B][S][H][hd]."""
    y = np.empty_like(x)
    for t in range(0, x.shape[1], 16):
        b = x[:, t:t + 16]
        s = np.abs(b).max(axis=(1, 3), keepdims=True) * float(np.float32(1 / 127))
        y[:, t:t + 16] = np.where(s > 0, np.rint(b / np.where(s > 0, s, 1)), 0) * s
    return y


def _oracle_logits(o, tokens, c, monkeypatch):
    plain = om.attention
    with monkeypatch.context() as m:
        m.setattr(om, "attention", lambda q, k, v, mode: plain(q, _as_cached(k), _as_cached(v), mode))
        return o.forward(np.asarray(tokens)[None], c=c, sign=0)[0]


def _prompts(shape, lens, seed=5):
    return [synth.uniform_tokens(1, n, shape.vocab, seed, 10 + i)[0].tolist() for i, n in enumerate(lens)]


@pytest.mark.parametrize("shape,mode", MODELS, ids=IDS)
def test_prompts_against_the_oracle(shape, mode, monkeypatch):
    """Ragged prompts in one call: the last token's logits.  Codes follow values that differ by the sums'
    order, so a few differ by one step (0.8% of a block's largest, of one token): 2e-3 for fp32; the
    framework's bar of 2e-2 for bf16."""
    o, g, c = _tuned(shape, mode)
    prompts = _prompts(shape, [1, 17, 40, 50])
    announce("prefill", shape.name, mode)
    ses = G.Session(g, 4, 64)
    got = host(ses.prefill([2, 0, 3, 1], prompts))
    ses.check()
    for i, p in enumerate(prompts):
        want = _oracle_logits(o, p, c, monkeypatch)[-1]
        _logits_close(got[i][None], want[None], 2e-3 if mode == "fp32" else 2e-2, f"prompt {i}")
    assert ses.cache.len.tolist() == [17, 50, 1, 40] == ses.lens


@pytest.mark.parametrize("shape,mode", MODELS, ids=IDS)
def test_tokens_after_prompts_against_the_oracle(shape, mode, monkeypatch):
    """Chunked prompts, then single tokens of all sequences: every step's logits.  A block that grows
    rounds its codes again with each new largest value (up to half a step each): the bar of 2e-2."""
    o, g, c = _tuned(shape, mode)
    full = _prompts(shape, [30, 9, 45], 6)
    want = [_oracle_logits(o, p, c, monkeypatch) for p in full]
    ses = G.Session(g, 3, 64, max_rows=16)
    announce("chunks and tokens", shape.name, mode)
    ses.prefill([0, 1, 2], [p[:-6] for p in full])
    for s in range(6, 0, -1):
        tok = torch.tensor([p[-s] for p in full], dtype=torch.int32, device=dev())
        got = host(ses.decode([0, 1, 2], tok))
        for i in range(3):
            _logits_close(got[i][None], want[i][len(full[i]) - s][None], 2e-2, f"step {s} sequence {i}")
    ses.check()


def test_int4_layers_of_few_rows_and_of_many_agree():
    """The same prompts through linear_rows (up to 64 rows) and through the two-halves linears (in one
    chunk of more): q s rounded to bf16 or not, within the framework's bar."""
    o, g, c = _tuned(LLAMA_S, "int4")
    prompts = _prompts(LLAMA_S, [33, 60, 21], 8)
    a = G.Session(g, 3, 64, max_rows=64).prefill([0, 1, 2], prompts)
    b = G.Session(g, 3, 64, max_rows=200).prefill([0, 1, 2], prompts)
    _logits_close(host(a), host(b), 2e-2, "few and many rows")


@pytest.mark.parametrize("mode", ["fp32", "int4"])
def test_forked_sequences_are_sequences_of_their_own(mode):
    shape = synth.TINY if mode == "fp32" else LLAMA_S
    _, g, _ = _tuned(shape, mode)
    p = _prompts(shape, [21], 9)[0]
    one, two = G.Session(g, 3, 128), G.Session(g, 3, 128)
    one.prefill([0], [p])
    one.prefill([1], [p])
    two.prefill([0], [p])
    two.fork([0], [1])
    rng = np.random.default_rng(0)
    for step in range(50):
        tok = torch.tensor(rng.integers(0, shape.vocab, 2), dtype=torch.int32, device=dev())
        x, y = one.decode([0, 1], tok), two.decode([0, 1], tok)
        assert torch.equal(x, y), step
        if step == 20:          # the two change places
            for s in (one, two):
                s.fork([1, 0], [0, 1])
    two.check()
    two.free([0])
    n = two.compact()
    assert n == 2 == int((two.cache.refs > 0).sum())
    # what is left goes on as before, in a smaller pool
    two.resize(3)
    one.free([0])
    for step in range(10):
        tok = torch.tensor(rng.integers(0, shape.vocab, 1), dtype=torch.int32, device=dev())
        assert torch.equal(one.decode([1], tok), two.decode([1], tok)), step
    one.check()
    two.check()


def test_generate_takes_the_likeliest_tokens():
    _, g, _ = _tuned(LLAMA_S, "int4")
    prompts = _prompts(LLAMA_S, [5, 70, 18], 11)
    out = g.generate(prompts, 6)
    ses = G.Session(g, 3, 80)
    logits = ses.prefill([0, 1, 2], prompts)
    for s in range(6):
        tok = logits.argmax(1).to(torch.int32)
        assert tok.tolist() == [o[s] for o in out]
        if s < 5:
            logits = ses.decode([0, 1, 2], tok)
    # the first sequence's third token as the end: it stops there, the others go on
    eos = out[0][2]
    cut = g.generate(prompts, 6, eos=eos)
    for a, b in zip(out, cut):
        assert b[:len(b)] == a[:len(b)] and eos not in b
    assert cut[0] == out[0][:out[0].index(eos)]


def test_beams_find_the_likeliest_pair():
    """As many beams as tokens: every pair of tokens is a candidate."""
    shape = synth.shrink(synth.TINY, vocab=32)
    _, g, _ = _tuned(shape, "fp32")
    prompts = _prompts(shape, [7, 12], 12)
    out = g.generate(prompts, 2, beams=32)
    for p, got in zip(prompts, out):
        ses = G.Session(g, 32, 64)
        first = torch.log_softmax(ses.prefill([0], [p])[0], 0)
        ses.fork([0] * 32, list(range(32)))
        second = torch.log_softmax(ses.decode(list(range(32)), torch.arange(32, dtype=torch.int32, device=dev())), 1)
        total = first[:, None] + second
        assert float(total[got[0], got[1]]) >= float(total.max()) - 1e-4
    assert all(len(x) <= 3 for x in g.generate(prompts, 3, beams=2, eos=out[0][0]))


def test_training_and_answering_take_turns():
    """A step between two answers changes them as a new session's; the step's losses are those without."""
    _, g, c = _tuned(LLAMA_S, "bf16")
    _, h, _ = _tuned(LLAMA_S, "bf16")
    tok = torch.from_numpy(synth.uniform_tokens(2, 32, LLAMA_S.vocab, 1, 2).astype(np.int32)).to(dev())
    p = _prompts(LLAMA_S, [20], 13)
    before = G.Session(g, 1, 64).prefill([0], p)
    for _ in range(3):
        x, y = g.step(tok, 5, 1e-3, 1e-2).clone(), h.step(tok, 5, 1e-3, 1e-2).clone()
        assert torch.equal(x, y)
        G.Session(g, 1, 64).prefill([0], p)
    assert torch.equal(g.arena.c, h.arena.c)
    a, b = G.Session(g, 1, 64).prefill([0], p), G.Session(h, 1, 64).prefill([0], p)
    assert torch.equal(a, b) and not torch.equal(a, before)


def test_too_few_pages_and_bad_calls():
    _, g, _ = _tuned(synth.TINY, "fp32")
    ses = G.Session(g, 2, 128, n_pages=2)
    ses.prefill([0], _prompts(synth.TINY, [100], 14))
    ses.prefill([1], _prompts(synth.TINY, [3], 14))
    with pytest.raises(RuntimeError, match="pages"):
        ses.check()
    assert ses.lens == [100, 0]
    with pytest.raises(ValueError):
        ses.resize(1)
    ses.resize(4)
    a = ses.prefill([1], _prompts(synth.TINY, [3], 14))
    ses.check()
    assert torch.equal(a, G.Session(g, 2, 128).prefill([1], _prompts(synth.TINY, [3], 14)))
    t = torch.zeros(1, dtype=torch.int32, device=dev())
    for bad in (lambda: ses.decode([2], t), lambda: ses.decode([-1], t), lambda: ses.decode([0, 0], t.repeat(2)),
                lambda: ses.decode([0], t.long()), lambda: ses.prefill([0], [[]]), lambda: ses.free([]),
                lambda: ses.prefill([0], [[1] * 29]), lambda: ses.fork([0, 1], [0]),
                lambda: G.generate(g, [], 3), lambda: g.generate([[1]], 0)):
        with pytest.raises(ValueError):
            bad()
    ses.check()
    assert ses.lens == ses.cache.len.tolist() == [100, 3]


def test_a_prompt_whose_middle_chunk_finds_no_page_has_no_hole():
    """Chunks of 100, 100 and 10 tokens where pages for the first alone are free: the last, which would fit behind the
    first, is not taken either, and the sequence goes on from what it holds."""
    _, g, _ = _tuned(synth.TINY, "fp32")
    p = _prompts(synth.TINY, [210], 15)[0]
    ses = G.Session(g, 2, 256, n_pages=3, max_rows=100)
    ses.prefill([0], [p])
    t = torch.zeros(1, dtype=torch.int32, device=dev())
    ses.decode([0], t)                       # (nor is anything else before the refusal is seen)
    ses.decode([1], t)
    with pytest.raises(RuntimeError, match="pages"):
        ses.check()
    assert ses.lens == ses.cache.len.tolist() == [100, 0]
    ses.check()
    ses.resize(8)
    got = ses.prefill([0], [p[100:]])
    ses.check()
    assert torch.equal(got, G.Session(g, 2, 256, max_rows=100).prefill([0], [p]))


def test_the_linear_hook_sees_every_launch_of_a_session():
    for mode, rows in (("int4", 3), ("int4", 70), ("bf16", 3)):
        _, g, _ = _tuned(LLAMA_S, mode)
        calls = []
        g.linear_hook = lambda stage, lin, T, flags: calls.append((stage, lin.d_in, lin.d_out, flags))
        G.Session(g, 1, 128).prefill([0], _prompts(LLAMA_S, [rows], 3))
        g.linear_hook = None
        per_layer = sum(isinstance(v, tuple) for v in g.layers[0].values())
        assert [c[0] for c in calls] == ["pre", "post"] * (per_layer * LLAMA_S.n_layers), (mode, rows)
        assert sum(c[3] == Z.EPI_SWIGLU for c in calls) == 2 * LLAMA_S.n_layers


def test_a_session_refuses_a_model_it_cannot_serve():
    """Heads of a width that the cache does not have, and a decoder without bases: before anything is reserved."""
    shape = synth.shrink(synth.TINY, n_heads=8, n_kv_heads=8)
    assert shape.head_dim not in (32, 64, 128)
    _, g, _ = _tuned(shape, "fp32")
    with pytest.raises(ValueError, match="head"):
        G.Session(g, 1, 64)
    _, g, _ = _tuned(synth.TINY, "fp32")
    ses = G.Session(g, 1, 64)
    ut, g.ut = g.ut, {}
    with pytest.raises(RuntimeError, match="basis"):
        ses.prefill([0], [[1, 2, 3]])
    g.ut = ut
    assert ses.lens == ses.cache.len.tolist() == [0]
    assert torch.equal(ses.prefill([0], [[1, 2, 3]]), G.Session(g, 1, 64).prefill([0], [[1, 2, 3]]))


def _plain_beams(g, prompt, n_new, beams, eos):
    """Beam search that runs every candidate from its prompt on, one sequence at a time.  Returns the best's tokens,
    whether a step's survivors were in another order than their parents, whether one had ended, and the smallest
    difference of scores that decided something."""
    ses = G.Session(g, 1, len(prompt) + n_new)

    def after(tokens):
        ses.free([0])
        logits = ses.prefill([0], [prompt])
        for t in tokens:
            logits = ses.decode([0], torch.tensor([t], dtype=torch.int32, device=dev()))
        ses.check()
        return torch.log_softmax(logits[0], 0).cpu().numpy().astype(np.float64)

    held, moved, ended, gap = [(0.0, [])], False, False, np.inf
    for step in range(n_new):
        if step and all(eos in t for _, t in held):
            break
        nxt = []
        for i, (score, t) in enumerate(held):
            if eos is not None and eos in t:
                nxt.append((score, t + [eos], i))
                ended = True
            else:
                nxt += [(score + float(p), t + [k], i) for k, p in enumerate(after(t))]
        nxt.sort(key=lambda c: -c[0])
        gap = min([gap] + [a[0] - b[0] for a, b in zip(nxt[:beams], nxt[1:beams + 1])])
        held = [c[:2] for c in nxt[:beams]]
        moved = moved or (step > 0 and [c[2] for c in nxt[:beams]] != list(range(beams)))
    best = held[0][1]
    return best[:best.index(eos)] if eos is not None and eos in best else best, moved, ended, gap


@pytest.mark.parametrize("beams", [2, 4])
def test_beams_of_several_steps_against_a_plain_search(beams):
    """Survivors in other orders than their parents, histories and ended candidates over five steps.  (The scores of
    two runs differ by the sums' order, some 1e-6: all decisions are by more.)"""
    shape = synth.shrink(synth.TINY, vocab=64)
    _, g, _ = _tuned(shape, "fp32")
    prompts = _prompts(shape, [9, 30], 23)
    plain = [_plain_beams(g, p, 5, beams, None) for p in prompts]
    assert all(p[1] for p in plain) and min(p[3] for p in plain) > 1e-4, [p[1:] for p in plain]
    assert g.generate(prompts, 5, beams=beams) == [p[0] for p in plain]
    eos = plain[0][0][1]
    cut = [_plain_beams(g, p, 5, beams, eos) for p in prompts]
    assert cut[0][2] and min(p[3] for p in cut) > 1e-4, [p[1:] for p in cut]
    assert g.generate(prompts, 5, beams=beams, eos=eos) == [p[0] for p in cut]


def test_trained_weights_are_those_of_the_training_products(monkeypatch):
    """With trained_weights no call of few rows takes q s: the same model as in calls of many rows."""
    o, g, c = _tuned(LLAMA_S, "int4")
    prompts = _prompts(LLAMA_S, [40, 37], 8)
    want = [_oracle_logits(o, p, c, monkeypatch)[-1] for p in prompts]
    many = G.Session(g, 2, 64).prefill([0, 1], prompts)          # 77 rows: the training forward's products
    monkeypatch.setattr(Z, "linear_rows", None)
    ses = G.Session(g, 2, 64, trained_weights=True)
    few = torch.cat([ses.prefill([i], [p]) for i, p in enumerate(prompts)])
    ses.check()
    _logits_close(host(few), np.stack(want), 2e-2, "oracle")
    err = float((few - many).norm() / many.norm())
    # sums in other orders, some of which round to the next bf16 activation: half the framework's bar
    assert err <= 1e-2, err
    out = g.generate(prompts, 3, trained_weights=True)
    assert [x[0] for x in out] == few.argmax(1).tolist()
