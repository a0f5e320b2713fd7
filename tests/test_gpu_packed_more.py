"""Packed sequences on the GPU where buffers, sizes and values are at their ends.  Tolerances as in test_gpu_packed."""
import pytest
import torch

import synth
from paper_2607_01125_amd import model as gm
from paper_2607_01125_amd import zoact as Z

from gpu_helpers import announce, dev
from test_gpu_model import LLAMA_S, _models
from test_gpu_packed import _texts

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
