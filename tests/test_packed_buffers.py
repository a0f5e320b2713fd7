"""What a Decoder keeps between packed batches of different sizes, without a GPU: the calls are replaced by notes of
their buffers."""
import weakref

import torch

import synth
from paper_2607_01125_amd import model as gm
from paper_2607_01125_amd import zoact as Z


def _decoder(**kw):
    d = gm.Decoder.__new__(gm.Decoder)
    d.__dict__.update(dict(dev=torch.device("cpu"), act=torch.bfloat16, r=8, _held=[], _proj_ws=None), **kw)
    return d


def test_packed_batches_share_one_pair_of_rotary_tables(monkeypatch):
    """Batches of many lengths: one pair of tables at a time, a graph's beside it, with the shorter tables' rows."""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    capturing = [False]
    shape = synth.shrink(synth.TINY, extra={"rope": dict(factor=4.0, original=16, low=1.0, high=2.0)})
    d = _decoder(s=shape, hd=shape.head_dim, _rope={}, _packed_rope=None)
    seen = []
    for n in (1, 17, 300, 256, 513, 1000, 40, 1025, 900):
        capturing[0] = n == 300
        cos, sin = d._packed_rope_tables(n)
        assert cos.shape[0] >= n and cos.shape == sin.shape
        want = Z.rope_tables(n, d.hd, shape.rope_theta, "cpu", **shape.extra["rope"])
        assert torch.equal(cos[:n], want[0]) and torch.equal(sin[:n], want[1])
        if not any(cos is r() for r in seen):
            seen.append(weakref.ref(cos))
        del cos, sin
    assert [None if r() is None else r().shape[0] for r in seen] == [None, 512, None, 2048] and not d._rope


def test_a_projections_partial_sums_outlive_larger_batches_for_a_graph(monkeypatch):
    """The workspace of a projection that a graph was captured on: a larger batch takes a new one, and the old one
    stays; without a capture it goes."""
    site, seen = (0, "down"), []
    d = _decoder(_adapted_sites={site}, ut={site: torch.zeros(8, 4096, dtype=torch.bfloat16)})
    monkeypatch.setattr(Z, "project", lambda x, ut, p, ws, n_all=None: seen.append(weakref.ref(ws)))
    capturing = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])

    def project(n):
        d._cur = {"p": torch.empty(n, 8, dtype=torch.bfloat16)}
        d._site(0, "down", torch.empty(n, 4096, dtype=torch.bfloat16), True, None)

    project(16)
    capturing[0] = True
    project(32)
    project(20)
    capturing[0] = False
    project(64)
    project(8)
    first, captured, smaller, larger, last = (r() for r in seen)
    assert first is None
    assert captured is not None and smaller is captured and larger is not captured and last is larger
    assert captured.numel() == Z.project_workspace_bytes(32, 4096, 8) > 0
