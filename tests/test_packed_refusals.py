"""What the calls of packed sequences and of the beam search refuse (no call here reaches the GPU), and the rotary
tables."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2607_01125_amd import model as gm
from paper_2607_01125_amd import zoact as Z

P, ODD = ctypes.c_void_p(256), ctypes.c_void_p(257)


def _seqs(**kw):
    f = dict(begin=256, n=3, rows=20)
    f.update(kw)
    return Z.PackedDesc(**f)


def _attend(s=None, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, H=4, Hkv=2, hd=64, scale=0.125, dt=Z.BF16, out=P):
    return Z.lib().zoact_attention_packed(ctypes.byref(s or _seqs()), q, ldq, k, ldk, v, ldv, H, Hkv, hd, scale, dt,
                                          out, None)


def _rope(x=P, ldx=256, out=P, ldo=256, dt=Z.BF16, rows=8, heads=4, hd=64, rot=64, layout=0, pos=P, cos=P, sin=P,
          n_pos=16):
    return Z.lib().zoact_rope_at(x, ldx, out, ldo, dt, rows, heads, hd, rot, layout, pos, cos, sin, n_pos, None)


def _xent(s=None, logits=P, tokens=P, V=100, loss=P, ws=P, nb=1 << 20):
    return Z.lib().zoact_xent_packed(logits, tokens, ctypes.byref(s or _seqs()), V, loss, ws, nb, None)


def _head(s=None, x=P, tokens=P, loss=P, ws=P, nb=1 << 40, **kw):
    f = dict(w_dtype=Z.BF16, w=256, d_in=64, d_out=64)
    f.update(kw)
    return Z.lib().zoact_linear_xent_packed(ctypes.byref(Z.LinearDesc(**f)), None, x, ctypes.byref(s or _seqs()), None,
                                            ctypes.byref(Z.pert_pair(0, 0, (0, 0), (0, 0), 0.0)), tokens, loss, ws, nb,
                                            None)


def _beams(logits=P, ldl=100, dt=Z.F32, ws=P, nb=1 << 40, **kw):
    f = dict(n=2, beams_in=3, beams=3, eos=2, vocab=100, length=4, score=256, hist=256, ld_hist=8, score_out=512,
             hist_out=512, ld_hist_out=8, token=256, src=256)
    f.update(kw)
    return Z.lib().zoact_beam_select(ctypes.byref(Z.BeamsDesc(**f)), logits, ldl, dt, ws, nb, None)


@pytest.mark.parametrize("s", [dict(begin=None), dict(begin=258), dict(n=0), dict(n=(1 << 24) + 1), dict(rows=-1),
                               dict(rows=2 ** 31 - 1023)])
def test_sequences_that_are_none(s):
    for f in (_attend, _xent, _head):
        assert f(_seqs(**s)) == Z.E_INVALID
        assert b"packed" in Z.lib().zoact_last_error()


@pytest.mark.parametrize("call", [
    lambda: _attend(q=None), lambda: _attend(out=None), lambda: _attend(k=ODD), lambda: _attend(ldq=255),
    lambda: _attend(ldk=127), lambda: _attend(ldv=0), lambda: _attend(H=3), lambda: _attend(H=0), lambda: _attend(Hkv=0),
    lambda: _attend(H=65536, Hkv=1, ldq=1 << 30), lambda: _attend(hd=0), lambda: _attend(hd=257, ldq=2000, ldk=2000, ldv=2000),
    lambda: _attend(scale=math.nan), lambda: _attend(scale=math.inf), lambda: _attend(dt=2),
    lambda: _attend(v=ctypes.c_void_p(258), dt=Z.F32),
    lambda: _rope(x=None), lambda: _rope(out=None), lambda: _rope(x=ODD), lambda: _rope(ldx=255), lambda: _rope(ldo=255),
    lambda: _rope(ldo=264), lambda: _rope(dt=2), lambda: _rope(rows=-1), lambda: _rope(rows=1 << 31), lambda: _rope(heads=0),
    lambda: _rope(heads=65535, hd=32769, ldx=1 << 32, ldo=1 << 32), lambda: _rope(hd=0), lambda: _rope(rot=0), lambda: _rope(rot=63), lambda: _rope(rot=66), lambda: _rope(layout=2),
    lambda: _rope(pos=ODD), lambda: _rope(cos=None), lambda: _rope(sin=ctypes.c_void_p(258)), lambda: _rope(n_pos=0),
    lambda: _rope(x=ctypes.c_void_p(258), dt=Z.F32),
    lambda: _xent(logits=None), lambda: _xent(tokens=None), lambda: _xent(loss=None), lambda: _xent(V=0),
    lambda: _xent(_seqs(rows=0)), lambda: _xent(tokens=ODD), lambda: _xent(ws=ctypes.c_void_p(260)),
    lambda: _head(tokens=None), lambda: _head(loss=None), lambda: _head(_seqs(rows=0)), lambda: _head(w_dtype=Z.F32),
    lambda: _head(d_in=60), lambda: _head(x=ODD),
    lambda: _beams(logits=None), lambda: _beams(score=None), lambda: _beams(score_out=None), lambda: _beams(hist_out=None),
    lambda: _beams(hist=None), lambda: _beams(dt=2), lambda: _beams(n=0), lambda: _beams(beams_in=0),
    lambda: _beams(beams_in=65), lambda: _beams(beams=0), lambda: _beams(beams=65, vocab=200, ldl=200),
    lambda: _beams(n=21846), lambda: _beams(vocab=2, ldl=2, eos=1), lambda: _beams(ldl=99), lambda: _beams(eos=100),
    lambda: _beams(eos=-2), lambda: _beams(length=-1), lambda: _beams(length=9, ld_hist_out=20),
    lambda: _beams(length=8), lambda: _beams(vocab=(1 << 30) + 1, ldl=1 << 31), lambda: _beams(token=258),
    lambda: _beams(score_out=256), lambda: _beams(hist_out=256), lambda: _beams(src=257), lambda: _beams(ws=ctypes.c_void_p(264)), lambda: _beams(logits=ctypes.c_void_p(258)),
])
def test_bad_arguments(call):
    assert call() == Z.E_INVALID
    assert Z.lib().zoact_last_error()


def test_workspaces_that_are_too_small():
    need = Z.beam_workspace_bytes(2, 3, 3, 100)
    assert need > 0 and _beams(nb=need - 1) == Z.E_WORKSPACE and _beams(ws=None) == Z.E_WORKSPACE
    assert Z.beam_workspace_bytes(2, 3, 65, 100) == 0 and Z.beam_workspace_bytes(0, 3, 3, 100) == 0
    assert _xent(nb=100) == Z.E_WORKSPACE and _xent(ws=None) == Z.E_WORKSPACE
    assert _head(nb=0) == Z.E_WORKSPACE and _head(ws=None) == Z.E_WORKSPACE


def test_no_rows_are_served_without_buffers():
    assert _attend(_seqs(rows=0), q=None, k=None, v=None, out=None) == Z.OK
    assert _rope(rows=0, x=None, out=None) == Z.OK
    assert _attend(_seqs(rows=0), H=3) == Z.E_INVALID and _rope(rows=0, rot=3) == Z.E_INVALID


def test_bindings_refuse_host_tensors_and_other_shapes():
    with pytest.raises(ValueError):
        Z.Packed(torch.zeros(3, dtype=torch.int32), 4, 4)
    with pytest.raises(ValueError):
        Z.Packed.of([3, -1], "cpu")
    with pytest.raises(ValueError):
        Z.Packed.of([], "cpu")
    for bad in ([], [[1, 2], []]):
        with pytest.raises(ValueError):
            gm.PackedBatch.of(bad, "cpu")


def test_tables_turn_by_the_formula():
    """Plain, slowed throughout, and slowed by parts: pairs that turn often within the trained length keep their
    pace, those that hardly turn go `factor` times slower."""
    f = 1.0e4 ** (-2.0 * np.arange(32) / 64)
    p = np.arange(300)[:, None]

    def near(got, ang, mag=1.0):
        # fp32 roundings of values of at most mag, and 2^-50 of an angle below 300
        for t, want in zip(got, (np.cos(ang), np.sin(ang))):
            assert np.abs(t.numpy().astype(np.float64) - mag * want).max() <= mag * (2.0 ** -24 + 2.0 ** -40)

    near(Z.rope_tables(300, 64, 1.0e4, "cpu"), p * f)
    near(Z.rope_tables(300, 64, 1.0e4, "cpu", factor=8.0), p * f / 8.0)
    turns = 2048 * f / (2 * np.pi)
    g = np.clip((turns - 1.0) / (4.0 - 1.0), 0, 1)
    assert (g == 0).any() and (g == 1).any() and ((g > 0) & (g < 1)).any()
    near(Z.rope_tables(300, 64, 1.0e4, "cpu", factor=8.0, original=2048, low=1.0, high=4.0, magnitude=1.25),
         p * (f * ((1 - g) / 8.0 + g)), 1.25)
    step = np.where(turns >= 3.0, 1.0, 1.0 / 8.0)
    near(Z.rope_tables(300, 64, 1.0e4, "cpu", factor=8.0, original=2048, low=3.0, high=3.0), p * f * step)
    for bad in (dict(n_pos=0), dict(rot_dim=63), dict(rot_dim=0), dict(factor=0.0), dict(low=2.0, high=1.0)):
        a = dict(n_pos=4, rot_dim=64, theta=1.0e4, device="cpu", factor=2.0)
        a.update(bad)
        with pytest.raises(ValueError):
            Z.rope_tables(a.pop("n_pos"), a.pop("rot_dim"), a.pop("theta"), **a)
