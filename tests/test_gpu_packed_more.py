"""Packed sequences on the GPU where buffers, sizes and values are at their ends.  Tolerances as in test_gpu_packed."""
import numpy as np
import pytest
import torch

import synth
from paper_2607_01125_amd import model as gm
from paper_2607_01125_amd import zoact as Z

import packed_ref as ref
from gpu_helpers import announce, dev, host, t_f32, t_i32
from test_gpu_model import LLAMA_S, _models
from test_gpu_packed import _act, _attend, _check, _draw, _qkv, _split, _texts

pytestmark = pytest.mark.gpu


def test_a_graph_of_deep_projections_outlives_larger_batches():
    """Layers deep enough that a projection's partial sums take a workspace: losses captured over a packed batch,
    replayed after larger batches have come, write into nothing else and give the eager values."""
    shape = synth.shrink(LLAMA_S, d_ff=2048)
    _, g = _models(shape, "bf16", 4)
    pert = Z.Pert(0, 0, 0, 0.0)
    batch = gm.PackedBatch.of(_texts(shape, [17, 40, 3]), dev())
    out = torch.zeros(2, device=dev())
    announce("packed graph, deep projections")
    g._loss_pair(batch, pert, out)
    want, ws = out.clone(), g._proj_ws
    assert ws is not None
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g._loss_pair(batch, pert, out)
    assert g._proj_ws is ws
    at, nbytes = ws.data_ptr(), ws.numel()
    del ws
    for lens in ([300, 200], [700, 1, 90]):
        other = torch.zeros(2, device=dev())
        g._loss_pair(gm.PackedBatch.of(_texts(shape, lens), dev()), pert, other)
        fresh = [torch.full((nbytes,), 7, dtype=torch.uint8, device=dev()) for _ in range(64)]
        assert all(f.data_ptr() != at for f in fresh)
        for _ in range(2):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        assert all(bool((f == 7).all()) for f in fresh)
    assert any(h.data_ptr() == at for h in g._held if isinstance(h, torch.Tensor))


@pytest.mark.parametrize("hd", [20, 24, 32, 64, 80, 128, 200])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_values_near_the_top_of_the_range(dt, hd):
    """Values of about 2^126, of one sign or of both: their weighted sums pass fp32's range, their means do not."""
    H, Hkv = 4, 2
    x, begin = _qkv([1, 150, 0, 333, 33], H, Hkv, hd, dt, seed=41, first=1, behind=2)
    v = _split(x, H, Hkv, hd)[2]
    v *= np.float32(2.0 ** 124)                # (exact in either type; below 2^127)
    assert np.nanmax(np.abs(v)) < 2.0 ** 127.5
    announce("attention_packed large values", dt, hd)
    for sign in (False, True):
        if sign:
            v[:] = np.abs(v)
        out = _attend(x, begin, H, Hkv, hd, dt, 0.1)
        _check(out, x, begin, H, Hkv, hd, dt, 0.1)
    assert np.nanmax(host(out)) > 2.0 ** 120


@pytest.mark.parametrize("hd", [32, 64, 80, 128])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_infinities_beside_large_values_and_masked_ones(dt, hd):
    """An infinity that rows see, beside values whose weighted sum passes the range on the other side, or beside a NaN
    that only later rows see: the formula's infinity; finite columns stay finite."""
    H, Hkv, L = 4, 2, 140
    x, begin = _qkv([L], H, Hkv, hd, dt, seed=42)
    v = _split(x, H, Hkv, hd)[2]
    v[:] = 1.0
    v[:, 0] = -2.0 ** 126
    v[10, 0] = np.inf
    v[10, 1], v[50, 1], v[60, 1] = np.inf, np.nan, -np.inf
    v[70, 2] = -np.inf
    v[:, 3] = 2.0 ** 127
    announce("attention_packed infinities beside large values", dt, hd)
    got = host(_attend(x, begin, H, Hkv, hd, dt, 0.02)).reshape(L, H, hd)[:, :H // Hkv]
    # means of equal values: a rounding of each weight and one of the mean in bf16; L + 64 of 2^-24 in fp32
    half = 2.0 ** -8 if dt == "bf16" else 2.0 ** -17
    assert np.all(np.abs(got[:10, :, 0] + 2.0 ** 126) <= half * 2.0 ** 127) and np.all(got[10:, :, 0] == np.inf)
    assert np.all(np.isfinite(got[:10, :, 1])) and np.all(got[10:50, :, 1] == np.inf) and np.isnan(got[50:, :, 1]).all()
    assert np.all(np.abs(got[:70, :, 2] - 1.0) <= 2 * half) and np.all(got[70:, :, 2] == -np.inf)
    assert np.all(np.abs(got[:, :, 3] - 2.0 ** 127) <= half * 2.0 ** 128)
    assert np.all(np.abs(got[:, :, 4:] - 1.0) <= 2 * half)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("hd", [24, 32, 64, 128])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_scores_whose_exponents_pass_the_range(dt, hd, sign):
    """Scores between 2^127 (1.5 and 1.98) of either sign, which log2(e) takes past fp32's range: the largest key's V
    and nothing else, or the mean of equal ones."""
    L = 150
    x = np.zeros((L, 3 * hd), np.float32)
    x[:, 0] = 2.0 ** 64
    x[:, hd] = sign * 2.0 ** 63 * (1.5 + (np.arange(L) * 37 % 32) / 66.0).astype(np.float32)
    x[:, hd] = synth.bf16_round(x[:, hd])
    x[:, 2 * hd:] = (np.arange(L * hd).reshape(L, hd) * 7919 % 128)
    begin = np.array([0, 64, L], np.int32)
    announce("attention_packed exponents past the range", dt, hd, sign)
    got = host(_attend(x, begin, 1, 1, hd, dt, 1.0))
    for b, e in zip(begin[:-1], begin[1:]):
        for t in range(b, e):
            s = x[b:t + 1, hd]
            want = x[b:t + 1, 2 * hd:][s == s.max()].astype(np.float64).mean(axis=0)
            # (values below 128: a rounding of the mean, and in fp32 some of the weights and sums)
            assert np.all(np.abs(got[t] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16), t


def test_positions_past_the_longest_sequence_are_refused():
    """A batch made by hand whose max_len is smaller than its positions reach, or whose positions are negative: the
    tables made for max_len would give other rows' angles.  One that fits gives what PackedBatch.of gives."""
    import dataclasses
    b = gm.PackedBatch.of(_texts(synth.TINY, [600, 3]), dev())
    announce("packed batch by hand")

    def made(max_len, pos):
        return gm.PackedBatch(b.tokens, dataclasses.replace(b.seqs, max_len=max_len), b.both, pos)

    for max_len, pos in ((599, b.pos), (256, b.pos), (0, b.pos), (600, b.pos + 1), (600, b.pos - 1)):
        with pytest.raises(ValueError, match="positions"):
            made(max_len, pos)
    _, g = _models(synth.TINY, "fp32", 4)
    pert = Z.Pert(0, 0, 0, 0.0)
    want = g.forward(b, pert).clone()
    for max_len in (600, 5000):
        assert torch.equal(g.forward(made(max_len, b.pos), pert), want)


@pytest.mark.parametrize("dt,hd,H,Hkv", [("bf16", 128, 4, 1), ("bf16", 64, 2, 2), ("bf16", 32, 4, 2), ("bf16", 80, 2, 1),
                                         ("fp32", 64, 2, 1), ("fp32", 128, 2, 2)])
def test_attention_of_thousands_of_tokens(dt, hd, H, Hkv):
    """A long sequence among short ones: whole tiles in their steady order, maxima that are followed late."""
    x, begin = _qkv([40, 3001, 7, 129], H, Hkv, hd, dt, seed=43, first=2, behind=3)
    announce("attention_packed long", dt, hd, H, Hkv)
    scale = float(np.float32(1 / np.sqrt(hd)))
    _check(_attend(x, begin, H, Hkv, hd, dt, scale), x, begin, H, Hkv, hd, dt, scale)


@pytest.mark.parametrize("heads,hd,rot", [(40, 128, 64), (40, 128, 128)])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [16411, 16412])
def test_rope_at_of_many_rows_in_pairs(rows, dt, heads, hd, rot):
    """So many rows that a thread takes two of them, an odd number among them; nothing behind the last is written."""
    n_pos = 300
    few = _draw((64, heads * hd), 1.0, 44, hd, rot, dt=dt)
    x = torch.empty(rows + 2, heads * hd, dtype=_act(few[:1], dt).dtype, device=dev())
    x[:rows] = _act(few, dt).repeat(rows // 64 + 1, 1)[:rows]
    x[rows:] = 9.0
    pos = synth.gen(44, rows).integers(-2, n_pos + 2, rows).astype(np.int32)
    cos, sin = (t.cpu().numpy() for t in Z.rope_tables(n_pos, rot, 1.0e4, "cpu"))
    out = torch.full_like(x, -7.0)
    announce("rope_at many rows", rows, dt, heads, hd, rot)
    for a, b in ((x, out), (x, x)):
        Z.rope_at(a[:rows], b[:rows], heads, hd, t_i32(pos), t_f32(cos), t_f32(sin), Z.ROPE_INTERLEAVED)
    assert torch.equal(out[:rows], x[:rows]) and bool((out[rows:] == -7.0).all()) and bool((x[rows:] == 9.0).all())
    half = 2.0 ** -8 if dt == "bf16" else 2.0 ** -24
    at = np.r_[0:5, 8000:8064, rows - 5:rows]
    want, bound = ref.turn(few[at % 64].astype(np.float64), heads, hd, rot, Z.ROPE_INTERLEAVED,
                           np.clip(pos[at], 0, n_pos - 1), cos, sin)
    assert np.all(np.abs(host(out[torch.from_numpy(at).to(dev())]) - want) <= half * np.abs(want) + bound)
