"""Packed sequences on the GPU against their formulas in float64: attention, rotary positions, losses, and whole
decoders over packed batches.

Tolerances, before the first run: outputs in bf16 are rounded once (2^-8 of the value) from probabilities rounded
to bf16 (2^-8 of each weight); fp32 ones 2^-24; fp32 sums as packed_ref states."""
import numpy as np
import pytest
import torch

import synth
from paper_2607_01125_amd import model as gm
from paper_2607_01125_amd import zoact as Z

import packed_ref as ref
from gpu_helpers import announce, assert_rel_close, dev, host, t_bf16, t_f32, t_i32
from test_gpu_model import LLAMA_S, OPT_S, _logits_close, _models

pytestmark = pytest.mark.gpu

BATCHES = {
    "one": [1], "edges": [0, 63, 1, 64, 0, 65, 127, 128, 129], "threes": [3] * 41, "long": [517], "two": [300, 211],
    "ones": [1] * 70, "wide": [259, 5, 31, 33, 257],
}


def _act(a, dt):
    return t_bf16(a) if dt == "bf16" else t_f32(a)


def _draw(shape, std, seed, *ids, dt):
    a = synth.normal(shape, std, seed, *ids)
    return synth.bf16_round(a) if dt == "bf16" else a


def _qkv(lens, H, Hkv, hd, dt, seed=1, first=0, behind=0, std=1.5):
    """A fused q|k|v buffer whose rows outside the sequences are NaN, on the host and on the device."""
    rows = first + sum(lens) + behind
    x = _draw((rows, (H + 2 * Hkv) * hd), std, seed, rows, H, hd, dt=dt)
    begin = ref.begins(lens, first)
    x[:begin[0]] = np.nan
    x[begin[-1]:] = np.nan
    return x, begin


def _split(x, H, Hkv, hd):
    a, b = H * hd, (H + Hkv) * hd
    return x[:, :a], x[:, a:b], x[:, b:]


def _attend(x, begin, H, Hkv, hd, dt, scale, out=None):
    t = _act(x, dt)
    rows = len(x)
    if out is None:
        out = torch.full((rows, H * hd), -7.0, dtype=t.dtype, device=dev())
    seqs = Z.Packed(t_i32(begin), rows, int(np.diff(begin).max()))
    Z.attention_packed(seqs, *_split(t, H, Hkv, hd), out, H, Hkv, hd, scale)
    return out


def _check(out, x, begin, H, Hkv, hd, dt, scale, rows=None, what=""):
    q, k, v = (a.astype(np.float64).reshape(len(x), -1, hd) for a in _split(x, H, Hkv, hd))
    want, bound, weight = ref.attention(q, k, v, begin, scale)
    got = host(out).reshape(want.shape)
    inside = np.zeros(len(x), bool)
    inside[begin[0]:begin[-1]] = True
    if rows is not None:
        inside &= rows
    else:
        assert np.all(got[~inside] == -7.0), "rows of no sequence were written"
    half = 2.0 ** -8 if dt == "bf16" else 2.0 ** -24
    tol = half * np.abs(want) + bound + (2.0 ** -8 * weight if dt == "bf16" else 0.0)
    got, want, tol = got[inside], want[inside], tol[inside]
    assert np.all(np.isfinite(got)), what
    over = np.abs(got - want) - tol
    assert over.max(initial=-1.0) <= 0, (what, np.unravel_index(over.argmax(), over.shape), over.max(), tol.max())


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("batch", sorted(BATCHES))
def test_attention(batch, dt, hd):
    for H, Hkv in ((4, 1), (4, 4), (14, 2), (6, 3)):
        announce("attention_packed", batch, dt, hd, H, Hkv)
        x, begin = _qkv(BATCHES[batch], H, Hkv, hd, dt, first=3, behind=5)
        scale = float(np.float32(1 / np.sqrt(hd)))
        _check(_attend(x, begin, H, Hkv, hd, dt, scale), x, begin, H, Hkv, hd, dt, scale, what=(H, Hkv))


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [1, 4, 8, 20, 24, 40, 80, 96, 120, 200, 256])
def test_attention_of_other_heads(hd, dt):
    announce("attention_packed any", hd, dt)
    x, begin = _qkv([1, 70, 0, 33], 4, 2, hd, dt, first=1, behind=1)
    _check(_attend(x, begin, 4, 2, hd, dt, 0.2), x, begin, 4, 2, hd, dt, 0.2)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_attention_of_strides_and_addresses_off_sixteen_bytes(dt):
    H, Hkv, hd = 4, 2, 64
    x, begin = _qkv([5, 100, 64], H, Hkv, hd, dt)
    t, rows = _act(x, dt), len(x)
    for pad, at in ((8, 8), (8, 4), (3, 0), (0, 1)):
        announce("attention_packed strides", dt, pad, at)
        qkv = []
        for a in _split(t, H, Hkv, hd):
            wide = torch.full((rows, a.shape[1] + pad + at), float("nan"), dtype=a.dtype, device=dev())
            wide[:, at:at + a.shape[1]] = a
            qkv.append(wide[:, at:at + a.shape[1]])
        out = torch.full((rows, H * hd), -7.0, dtype=t.dtype, device=dev())
        Z.attention_packed(Z.Packed(t_i32(begin), rows, 100), *qkv, out, H, Hkv, hd, 0.125)
        _check(out, x, begin, H, Hkv, hd, dt, 0.125, what=(pad, at))


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_attention_of_other_scales(dt, scale):
    """Weights all alike, the smallest product first, and far apart."""
    announce("attention_packed scale", dt, scale)
    x, begin = _qkv([130, 77], 4, 2, 64, dt, seed=3)
    _check(_attend(x, begin, 4, 2, 64, dt, scale), x, begin, 4, 2, 64, dt, scale)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_attention_of_rising_scores(dt):
    """The running maximum moves at every key, by small and by large steps; rows of equal scores."""
    H, Hkv, hd, L = 4, 2, 64, 400
    x, begin = _qkv([L, 40], H, Hkv, hd, dt, seed=4)
    q, k, v = _split(x, H, Hkv, hd)
    q[:] = 0.0
    k[:] = 0.0
    q[:, ::hd] = 4.0
    k[:L, ::hd] = _round((np.arange(L) * 0.11)[:, None] * np.array([[1.0, 3.0]]), dt)
    announce("attention_packed rising", dt)
    _check(_attend(x, begin, H, Hkv, hd, dt, 0.5), x, begin, H, Hkv, hd, dt, 0.5)


def _round(a, dt):
    a = np.asarray(a, np.float32)
    return synth.bf16_round(a) if dt == "bf16" else a


@pytest.mark.parametrize("hd", [24, 32, 64, 80, 128])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_a_row_may_not_attend_to_does_not_reach_it(bad, dt, hd):
    """Keys and values of later tokens, and of other sequences, that are not finite: rows before them are what they
    would be without.  (Rows from them on are the formula's NaN or infinities.)"""
    H, Hkv = 4, 2
    lens = [100, 150, 7, 64]
    x, begin = _qkv(lens, H, Hkv, hd, dt, seed=5)
    clean = x.copy()
    rows = np.ones(len(x), bool)
    _, k, v = _split(x, H, Hkv, hd)
    for seq, at in ((1, 37), (1, 100), (3, 63), (2, 1)):
        t = begin[seq] + at
        k[t, 0] = bad
        v[t, hd - 1:hd + 1] = bad
        rows[t:begin[seq + 1]] = False
    v[begin[1] + 70:begin[1] + 72] = bad
    rows[begin[1] + 70:begin[2]] = False
    announce("attention_packed masked", bad, dt, hd)
    scale = float(np.float32(1 / np.sqrt(hd)))
    out = _attend(x, begin, H, Hkv, hd, dt, scale)
    _check(out, clean, begin, H, Hkv, hd, dt, scale, rows=rows)
    # a value that is not finite reaches every later row of its heads and column
    got = host(out).reshape(len(x), H, hd)
    after = got[begin[1] + 100:begin[2], :2, hd - 1]
    assert not np.isfinite(after).any()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_scores_of_minus_infinity_have_no_weight(dt):
    """A key whose product with every query is -inf (by its first value) adds nothing, also where it is the first;
    a row that has nothing else is the formula's NaN."""
    H, Hkv, hd, L = 2, 1, 64, 150
    x, begin = _qkv([L], H, Hkv, hd, dt, seed=6)
    q, k, v = _split(x, H, Hkv, hd)
    q[:, ::hd] = 1.0
    gone = np.r_[0:70, 80, 130:140]
    kept = np.setdiff1d(np.arange(L), gone)
    k[gone, 0] = -np.inf
    announce("attention_packed -inf", dt)
    got = host(_attend(x, begin, H, Hkv, hd, dt, 0.125)).reshape(L, H, hd)
    assert np.isnan(got[:70]).all()
    y = x[kept]
    want, bound, weight = ref.attention(*(a.astype(np.float64).reshape(len(y), -1, hd) for a in _split(y, H, Hkv, hd)),
                                        np.array([0, len(y)]), 0.125)
    half = 2.0 ** -8 if dt == "bf16" else 2.0 ** -24
    tol = half * np.abs(want) + bound + (2.0 ** -8 * weight if dt == "bf16" else 0.0)
    assert np.all(np.abs(got[kept] - want) <= tol)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_bounds_that_do_not_ascend(dt):
    """Bounds outside the rows, or that descend, touch nothing else."""
    H, Hkv, hd = 4, 2, 64
    x, _ = _qkv([300, 20], H, Hkv, hd, dt)
    for wrong in ([0, 300, 400], [-5, 300, 320], [200, 100, 320], [400, 500, 600], [0, 320, 0],
                  [0, 320] * 100):
        announce("attention_packed bad bounds", dt, wrong[:4])
        guard = torch.full((3 * 320, H * hd), -7.0, dtype=_act(x[:1], dt).dtype, device=dev())
        out = guard[320:640]
        _attend(x, np.array(wrong, np.int32), H, Hkv, hd, dt, 0.125, out=out)
        g = host(guard)
        assert np.all(g[:320] == -7.0) and np.all(g[640:] == -7.0)


@pytest.mark.parametrize("Hkv", [1, 4])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [62, 63, 64, 65, 129, 4097])
def test_many_sequences(n, dt, Hkv):
    """Numbers of sequences around those that one read of the bounds covers, most of them a few rows or none."""
    H, hd = 4, 32
    lens = [(i * 7919) % 6 for i in range(n)]
    lens[n // 2], lens[n - 1] = 70, 41
    x, begin = _qkv(lens, H, Hkv, hd, dt, seed=n, first=3, behind=2)
    announce("attention_packed many", n, dt, Hkv)
    _check(_attend(x, begin, H, Hkv, hd, dt, 0.2), x, begin, H, Hkv, hd, dt, 0.2)


def test_as_many_sequences_as_are_allowed():
    """2^24 sequences of one row (more workgroups than one launch has in the tiles' kernel): each row is its V."""
    n, hd = 1 << 24, 32
    v = torch.randint(-100, 100, (n, hd), device=dev(), dtype=torch.int8).to(torch.bfloat16)
    out = torch.zeros_like(v)
    announce("attention_packed 2^24 sequences")
    seqs = Z.Packed(torch.arange(n + 1, device=dev(), dtype=torch.int32), n, 1)
    Z.attention_packed(seqs, v, v, v, out, 1, 1, hd, 0.01)
    assert torch.equal(out, v)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_scores_near_the_ends_of_the_range(dt):
    """Scores between -1e38 and -2.2e38, far apart: the largest key's V and nothing else; and a scale whose product
    with log2(e) is not finite, with scores of 0: the mean."""
    L, hd = 150, 64
    x = np.zeros((L, 3 * hd), np.float32)
    x[:, 0] = 2.0 ** 63
    x[:, hd] = -2.0 ** 63 * (1.25 + (np.arange(L) * 37 % 64) / 64.0)           # (exact in bf16; each score at most twice)
    x[:, 2 * hd:] = (np.arange(L * hd).reshape(L, hd) * 7919 % 128)
    begin = np.array([0, 64, L], np.int32)
    announce("attention_packed ends of the range", dt)
    got = host(_attend(x, begin, 1, 1, hd, dt, 1.0))
    for b, e in zip(begin[:-1], begin[1:]):
        for t in range(b, e):
            s = x[b:t + 1, hd]
            assert np.array_equal(got[t], x[b:t + 1, 2 * hd:][s == s.max()].mean(axis=0)), t
    x[:, 0] = 0.0
    _check(_attend(x, begin, 1, 1, hd, dt, 3.0e38), x, begin, 1, 1, hd, dt, 3.0e38)


# ------------------------------------------------------------------ offsets past 32 bits
@pytest.mark.parametrize("dt,hd", [("bf16", 64), ("fp32", 64), ("bf16", 24), ("bf16", 20)])
def test_attention_and_rotary_past_two_to_the_31_values(dt, hd):
    """A sequence at the end of tensors of more than 2^31 values, and rows turned there: as at the beginning."""
    H, Hkv, n = 8, 1, 150
    width = (H + 2 * Hkv) * hd
    rows = -(-(2 ** 31 + 2 ** 20) // width) + n
    small, _ = _qkv([n], H, Hkv, hd, dt, seed=31)
    few = _act(small, dt)
    x = torch.zeros(rows, width, dtype=few.dtype, device=dev())
    x[rows - n:] = few
    announce("attention_packed past 2^31", dt, hd)
    out = torch.empty(rows, H * hd, dtype=few.dtype, device=dev())
    near = torch.empty(n, H * hd, dtype=few.dtype, device=dev())
    Z.attention_packed(Z.Packed(t_i32([rows - n, rows]), rows, n), *_split(x, H, Hkv, hd), out, H, Hkv, hd, 0.2)
    Z.attention_packed(Z.Packed.of([n], dev()), *_split(few, H, Hkv, hd), near, H, Hkv, hd, 0.2)
    # (the same rows of a sequence in a workgroup, whose order of work alone differs)
    assert torch.equal(out[rows - n:], near)
    cos, sin = Z.rope_tables(64, hd, 1.0e4, dev())
    pos = torch.full((rows,), 3, dtype=torch.int32, device=dev())
    Z.rope_at(x, x, H + 2 * Hkv, hd, pos, cos, sin)
    Z.rope_at(few, few, H + 2 * Hkv, hd, pos[:n], cos, sin)
    assert torch.equal(x[rows - n:], few)


def test_losses_past_two_to_the_31_logits():
    V = 2 ** 29 + 4
    lg = torch.zeros(2, 3, V, device=dev())
    lg[1, 1, V - 1] = 7.0
    loss, ws = torch.empty(2, device=dev()), torch.empty(Z.loss_workspace_bytes(), dtype=torch.uint8, device=dev())
    announce("xent_packed past 2^31")
    Z.xent_packed(lg, t_i32([0, 1, V - 1]), Z.Packed.of([3], dev()), loss, ws)
    # two rows each of log V; one logit of 7 takes 3.5 of the mean (and adds 1100 to a sum of 5e8: 2e-6)
    want = np.log(float(V)) - np.array([0.0, 3.5])
    assert np.abs(host(loss) - want).max() < 1e-4


# ------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("layout", [Z.ROPE_HALF, Z.ROPE_INTERLEAVED])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,rot", [(128, 128), (128, 64), (64, 64), (32, 16), (80, 24), (40, 10), (5, 2), (7, 6)])
def test_rope_at(hd, rot, dt, layout):
    heads, rows, n_pos = 3, 67, 50
    x = _draw((rows, heads * hd), 1.0, 7, hd, rot, dt=dt)
    pos = synth.gen(1, hd).integers(-4, n_pos + 4, rows).astype(np.int32)       # some past either end
    cos, sin = (t.cpu().numpy() for t in Z.rope_tables(n_pos, rot, 1.0e4, "cpu", magnitude=1.1))
    half = 2.0 ** -8 if dt == "bf16" else 2.0 ** -24
    for pad, at, given in ((0, 0, True), (8, 0, False), (5, 1, True)):
        p = np.clip(pos if given else np.arange(rows), 0, n_pos - 1)
        want, bound = ref.turn(x.astype(np.float64), heads, hd, rot, layout, p, cos, sin)
        wide = torch.full((rows, heads * hd + pad + at), 9.0, dtype=_act(x, dt).dtype, device=dev())
        xs = wide[:, at:at + heads * hd]
        xs.copy_(_act(x, dt))
        out = torch.full((rows, heads * hd), -7.0, dtype=wide.dtype, device=dev())
        announce("rope_at", hd, rot, dt, layout, pad, at)
        tp = t_i32(pos) if given else None
        Z.rope_at(xs, out, heads, hd, tp, t_f32(cos), t_f32(sin), layout)
        Z.rope_at(xs, xs, heads, hd, tp, t_f32(cos), t_f32(sin), layout)        # in place
        assert np.array_equal(host(out), host(xs)) and (host(wide)[:, heads * hd + at:] == 9.0).all()
        assert np.all(np.abs(host(out) - want) <= half * np.abs(want) + bound)


def test_rope_at_gives_what_rope_gives():
    """The rectangular call's rows, at their positions: the same values."""
    heads, hd, seq, n = 5, 128, 33, 3
    cos, sin = Z.rope_tables(seq, hd, 5.0e5, dev())
    for dt in ("bf16", "fp32"):
        x = _act(_draw((n * seq, heads * hd), 1.0, 8, dt=dt), dt)
        y, pos = x.clone(), torch.arange(n * seq, dtype=torch.int32, device=dev()) % seq
        announce("rope_at and rope", dt)
        Z.rope(y, 0, heads, hd, seq, cos, sin)
        Z.rope_at(x, x, heads, hd, pos, cos, sin)
        # (two fp32 evaluations, then one rounding each)
        tol = 2.0 ** -7 if dt == "bf16" else 2.0 ** -22
        assert np.all(np.abs(host(x) - host(y)) <= tol * np.abs(host(y)) + 2.0 ** -21)


# ------------------------------------------------------------------ losses
@pytest.mark.parametrize("lens,V", [([1, 0, 5, 2, 64, 1], V) for V in (1, 5, 512, 2048, 2051, 16391)]
                         + [([3000, 1, 2200], 40), ([1100, 900], 2050)])
def test_xent_from_logits(lens, V):
    """fp32 sums of exponentials: a thread's chain and the joins are below 60 roundings by 2^-24, an exponential is
    within 2^-20 (__expf of arguments down to -30); the logits are at most 20: below 1e-5 in all."""
    begin = ref.begins(lens, 2)
    rows = int(begin[-1]) + 3
    lg = synth.normal((2, rows, V), 3.0, 9, V)
    lg[:, :2], lg[:, begin[-1]:] = np.nan, np.nan
    tok = synth.gen(2, V).integers(-1, V + 1, rows).astype(np.int32)       # ids outside are clamped
    loss = torch.empty(2, device=dev())
    ws = torch.empty(Z.loss_workspace_bytes(), dtype=torch.uint8, device=dev())
    announce("xent_packed", lens, V)
    Z.xent_packed(t_f32(lg), t_i32(tok), Z.Packed(t_i32(begin), rows, 64), loss, ws)
    want = [ref.loss(lg[h].astype(np.float64), tok, begin) for h in range(2)]
    assert np.all(np.abs(host(loss) - want) <= 1e-5 * (1 + np.abs(want))), (host(loss), want)


@pytest.mark.parametrize("lens,V,d", [([1, 9, 0, 40, 2], 512, 128), ([130, 1, 200], 1008, 256), ([2], 64, 128)])
def test_xent_in_the_heads_epilogue(lens, V, d):
    begin = ref.begins(lens)
    rows = int(begin[-1])
    x = synth.bf16_round(synth.normal((2, rows, d), 1.0, 10, V))
    w = synth.bf16_round(synth.normal((V, d), 0.1, 11, V))
    tok = synth.gen(3, V).integers(0, V, rows).astype(np.int32)
    layer = Z.Linear(t_bf16(w), d, V)
    ws = torch.empty(Z.linear_xent_workspace_bytes(rows, V), dtype=torch.uint8, device=dev())
    loss = torch.empty(2, device=dev())
    announce("linear_xent_packed", lens, V, d)
    Z.linear_xent_packed(layer, None, t_bf16(x), t_i32(tok), Z.Packed(t_i32(begin), rows, max(lens)), None,
                         Z.Pert(0, 0, 0, 0.0), loss, ws)
    want = [ref.loss(x[h].astype(np.float64) @ w.astype(np.float64).T, tok, begin) for h in range(2)]
    # (logits: d fp32 roundings of sums below 10; the rest as from logits)
    assert np.all(np.abs(host(loss) - want) <= 2e-5 * (1 + np.abs(want))), (host(loss), want)


def test_a_batch_without_a_next_token_has_no_loss():
    loss = torch.zeros(2, device=dev())
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev())
    announce("loss of ones")
    Z.xent_packed(torch.zeros(2, 3, 8, device=dev()), t_i32([0, 1, 2]), Z.Packed.of([1, 1, 1], dev()), loss, ws)
    assert np.isnan(host(loss)).all()
    x = torch.zeros(2, 1, 128, dtype=torch.bfloat16, device=dev())
    layer = Z.Linear(torch.zeros(64, 128, dtype=torch.bfloat16, device=dev()), 128, 64)
    loss.zero_()
    ws = torch.empty(Z.linear_xent_workspace_bytes(1, 64), dtype=torch.uint8, device=dev())
    Z.linear_xent_packed(layer, None, x, t_i32([3]), Z.Packed.of([1], dev()), None, Z.Pert(0, 0, 0, 0.0), loss, ws)
    assert np.isnan(host(loss)).all()


# ------------------------------------------------------------------ whole decoders
MODELS = [(synth.TINY, "fp32"), (LLAMA_S, "bf16"), (LLAMA_S, "int4"), (OPT_S, "bf16")]


def _texts(shape, lens, seed=5):
    return [synth.uniform_tokens(1, n, shape.vocab, seed, 20 + i)[0] for i, n in enumerate(lens)]


@pytest.mark.parametrize("shape,mode", MODELS, ids=lambda x: getattr(x, "name", x))
def test_a_packed_step_against_the_oracle(shape, mode):
    """Both halves' logits of every sequence, the losses, and a step: the bars of the rectangular forward (2e-2 for
    bf16, 1e-4 for fp32)."""
    o, g = _models(shape, mode, 4, perturb=True)
    c = synth.normal((o.k,), 0.05, 4, 77)
    c = synth.bf16_round(c) if g.c_bf16 else c
    g.arena.c.copy_(torch.from_numpy(c))
    eps, texts = 1e-2, _texts(shape, [17, 1, 40, 2, 33])
    batch = gm.PackedBatch.of(texts, dev())
    announce("packed step", shape.name, mode)
    got = host(g.forward(batch, Z.Pert(3, 1, 0, eps)))
    bar = 1e-4 if mode == "fp32" else 2e-2
    losses = []
    for h, sign in enumerate((1, -1)):
        total, count, r0 = 0.0, 0, 0
        for t in texts:
            want = o.forward(t[None], c=c, sign=sign, eps=eps, z_ctx=(3, 1, 0))[0]
            _logits_close(got[h, r0:r0 + len(t)], want, bar, f"half {h}, sequence at {r0}")
            total += ref.loss(want, t, [0, len(t)]) * (len(t) - 1) if len(t) > 1 else 0.0
            count += len(t) - 1
            r0 += len(t)
        losses.append(total / count)
    assert_rel_close(host(g.losses(batch, 3, 1, eps)), losses, bar, "losses")
    before = g.arena.c.clone()
    loss = g.step(batch, 3, eps, 1e-3)
    assert_rel_close(host(loss), losses, bar, "losses of the step")
    assert not torch.equal(before, g.arena.c) and int(g.status) == 0
    # a rectangular batch after it, and the packed form of the same batch
    toks = synth.uniform_tokens(4, 12, shape.vocab, 6, 1)
    rect = host(g.losses(t_i32(toks), 3, 2, eps)).copy()
    assert_rel_close(host(g.losses(gm.PackedBatch.of(list(toks), dev()), 3, 2, eps)), rect, bar, "packed and rectangular")


def test_packed_batches_that_do_not_fit():
    b = gm.PackedBatch.of([[1, 2, 3], [4]], dev())
    _, g = _models(synth.TINY, "fp32", 4)
    for bad in (dict(tokens=b.tokens[:3]), dict(pos=b.pos[:4]), dict(both=b.seqs), dict(tokens=b.tokens.long()),
                dict(tokens=b.tokens.cpu())):
        f = dict(tokens=b.tokens, seqs=b.seqs, both=b.both, pos=b.pos)
        f.update(bad)
        with pytest.raises(ValueError):
            gm.PackedBatch(**f)
    with pytest.raises(ValueError):
        g.forward(b, Z.Pert(0, 0, 0, 0.0), distinct_halves=True)


@pytest.mark.parametrize("mode", ["fp32", "bf16"])
def test_a_packed_forward_in_a_graph_outlives_larger_batches(mode):
    """Losses captured over a packed batch, replayed after larger packed and other batches have come: the eager
    values."""
    _, g = _models(LLAMA_S if mode == "bf16" else synth.TINY, mode, 4)
    shape, pert = g.s, Z.Pert(0, 0, 0, 0.0)
    batch = gm.PackedBatch.of(_texts(shape, [17, 40, 3]), dev())
    out = torch.zeros(2, device=dev())
    announce("packed graph", mode)
    g._loss_pair(batch, pert, out)
    want = out.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g._loss_pair(batch, pert, out)
    for lens in ([300, 200], [700, 1, 90]):
        larger = gm.PackedBatch.of(_texts(shape, lens), dev())
        other = torch.zeros(2, device=dev())
        g._loss_pair(larger, pert, other)
        kept = other.clone()
        fresh = [torch.full((1 << 16,), 7.0, device=dev()) for _ in range(64)]   # (what was freed is used again)
        for _ in range(2):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        g._loss_pair(larger, pert, other)
        assert torch.equal(other, kept) and all(bool((f == 7.0).all()) for f in fresh)


def test_packed_query_steps_and_calibration():
    """step_q over a packed batch, and bases from packed calibration text."""
    o, g = _models(LLAMA_S, "bf16", 5)
    batch = gm.PackedBatch.of(_texts(LLAMA_S, [9, 30, 4], 8), dev())
    announce("packed step_q")
    losses = host(g.step_q(batch, 7, 1e-2, 1e-3, 3))
    assert losses.shape == (4,) and np.isfinite(losses).all() and int(g.status) == 0
    text = gm.PackedBatch.of(_texts(LLAMA_S, [100, 33, 260, 7], 9), dev())
    announce("packed calibration")
    sites = {}
    g.forward(text, Z.Pert(0, 0, 0, 0.0), calibrate=lambda l, s, x: sites.setdefault((l, s), x[:400].float().clone()))
    g.basis_init(text, Z.EigOpts(tol=1e-4, adaptive=1))
    for key in g.site_dims():
        u, x = g.ut[key].float(), sites[key]
        gram = (x.double().T @ x.double())
        best = torch.linalg.eigvalsh(gram)[-g.r:].sum()
        held = torch.trace(u.double() @ gram @ u.double().T)
        # the basis holds what the top directions hold (bf16 columns: 2^-7 of it)
        assert float(held / best) > 1 - 2.0 ** -6, key


def test_scaled_positions_reach_every_forward():
    """A model whose positions are scaled: the packed and the rectangular forward and the cache's tokens agree, and
    differ from the unscaled model's by more than ten times the bar of the first two."""
    wide = synth.shrink(synth.TINY, init_std=0.1)        # (weights that make attention matter)
    shape = synth.shrink(wide, extra={"rope": dict(factor=4.0, original=16, low=1.0, high=2.0)})
    _, g = _models(shape, "fp32", 4)
    _, p = _models(wide, "fp32", 4)
    text = _texts(shape, [48], 11)[0]
    pert = Z.Pert(0, 0, 0, 0.0)
    announce("scaled positions")
    got = host(g.forward(gm.PackedBatch.of([text, text], dev()), pert))[0]
    rect = host(g.forward(t_i32(np.stack([text, text])), pert))[0]
    _logits_close(got.reshape(rect.shape)[0], rect[0], 1e-4, "packed and rectangular")
    plain = host(p.forward(t_i32(np.stack([text, text])), pert))[0]
    assert np.linalg.norm(plain[0] - rect[0]) > 1e-3 * np.linalg.norm(rect[0])
    from paper_2607_01125_amd import generate as G
    ses = G.Session(g, 1, 64)
    last = host(ses.prefill([0], [text.tolist()]))
    other = host(G.Session(p, 1, 64).prefill([0], [text.tolist()]))
    # (keys and values in 8 bits: nearer to its own forward than to the unscaled cache's)
    assert np.linalg.norm(last - rect[0, -1:]) < 0.5 * np.linalg.norm(last - other)


# ------------------------------------------------------------------ graphs and streams
def test_a_run_of_them_from_a_graph():
    """Rotary, attention and loss in one graph, replayed with other inputs and other lengths: the eager values."""
    H, Hkv, hd, V = 4, 2, 64, 512
    rows = 200
    x = torch.empty(rows, (H + 2 * Hkv) * hd, dtype=torch.bfloat16, device=dev())
    begin = torch.zeros(5, dtype=torch.int32, device=dev())
    pos = torch.zeros(rows, dtype=torch.int32, device=dev())
    tok = torch.zeros(rows, dtype=torch.int32, device=dev())
    out = torch.zeros(rows, H * hd, dtype=torch.bfloat16, device=dev())
    cos, sin = Z.rope_tables(256, hd, 1.0e4, dev())
    layer = Z.Linear(t_bf16(synth.bf16_round(synth.normal((V, H * hd), 0.1, 12, 1))), H * hd, V)
    ws = torch.empty(Z.linear_xent_workspace_bytes(rows // 2, V), dtype=torch.uint8, device=dev())
    loss = torch.zeros(2, device=dev())
    half = Z.Packed(torch.tensor([0, 30, 100], dtype=torch.int32, device=dev()), rows // 2, 100)
    seqs = Z.Packed(begin, rows, rows)

    def go():
        turned = x[:, :(H + Hkv) * hd]
        Z.rope_at(turned, turned, H + Hkv, hd, pos, cos, sin)
        Z.attention_packed(seqs, *_split(x, H, Hkv, hd), out, H, Hkv, hd, 0.125)
        Z.linear_xent_packed(layer, None, out, tok[:rows // 2], half, None, Z.Pert(0, 0, 0, 0.0), loss, ws)

    def load(seed, lens):
        x.copy_(t_bf16(synth.bf16_round(synth.normal(tuple(x.shape), 1.0, 13, seed))))
        begin.copy_(t_i32(ref.begins(lens)))
        pos.copy_(t_i32(np.concatenate([np.arange(n) for n in lens])))
        tok.copy_(t_i32(synth.uniform_tokens(1, rows, V, 13, seed)[0]))
        out.zero_()
        loss.zero_()

    load(0, [50, 50, 60, 40])
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for seed, lens in ((1, [200, 0, 0, 0]), (2, [1, 64, 65, 70]), (3, [50, 50, 50, 50])):
        announce("graph", seed)
        load(seed, lens)
        go()
        want = out.clone(), loss.clone()
        torch.cuda.synchronize()
        for _ in range(2):
            load(seed, lens)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(loss, want[1]) and bool(torch.isfinite(loss).all())


def test_calls_on_another_stream_wait_for_it_only():
    H, Hkv, hd = 4, 2, 64
    x, begin = _qkv([90, 30], H, Hkv, hd, "bf16", seed=14)
    s = torch.cuda.Stream()
    announce("other stream")
    t, b = _act(x, "bf16"), t_i32(begin)
    out = torch.full((len(x), H * hd), -7.0, dtype=torch.bfloat16, device=dev())
    torch.cuda.synchronize()
    Z.attention_packed(Z.Packed(b, len(x), 90), *_split(t, H, Hkv, hd), out, H, Hkv, hd, 0.125, stream=s)
    s.synchronize()
    _check(out, x, begin, H, Hkv, hd, "bf16", 0.125)
