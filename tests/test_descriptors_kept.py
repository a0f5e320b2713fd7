"""What linear_rows and the cache's calls keep of their arguments between calls: an address is used again only while
the tensor that it was taken from is still there (CPU tensors, device -1: no call is made)."""
import copy
import gc
import weakref

import pytest
import torch

from paper_2607_01125_amd import zoact as Z


def _layer():
    return Z.Linear(torch.zeros(64, 128, dtype=torch.uint8), 256, 64, 8, bias=torch.zeros(64, dtype=torch.bfloat16),
                    w_scales=torch.zeros(64, 2, dtype=torch.bfloat16), ws=torch.zeros(4096, dtype=torch.uint8))


def _moves(t):
    """Ways in which a tensor gets other memory without being another tensor."""
    def by_data():
        t.data = t.detach().clone()

    def by_set():
        t.set_(t.detach().clone())

    def by_resize():
        n = t.numel()
        t.resize_(1 << 20)
        t.resize_(n)

    return by_data, by_set, by_resize


@pytest.mark.parametrize("how", range(3))
@pytest.mark.parametrize("field", ["w", "w_scales", "bias", "ws"])
def test_a_layer_whose_tensor_moves(field, how):
    lin = _layer()
    first = lin.rows_ref(-1)
    assert lin.rows_ref(-1) is first
    t = getattr(lin, field)
    shape, old = t.shape, t.data_ptr()
    keep = t.detach()                                    # (so that the old memory is not handed out again)
    _moves(t)[how]()
    assert t.data_ptr() != old
    if t.shape != shape and field != "ws":
        with pytest.raises(ValueError):
            lin.rows_ref(-1)
        t.resize_(shape)
    d = lin.rows_ref(-1)._obj
    assert getattr(d, field) == t.data_ptr() and keep is not None
    assert (d.w, d.w_scales, d.bias, d.ws) == tuple(x.data_ptr() for x in (lin.w, lin.w_scales, lin.bias, lin.ws))


def test_a_layer_whose_fields_change():
    lin = _layer()
    lin.rows_ref(-1)
    lin.r = 16
    assert lin.rows_ref(-1)._obj.r == 16
    lin.coef_offset, lin.plain = 24, (16, 32)
    d = lin.rows_ref(-1)._obj
    assert (d.coef_offset, d.plain_begin, d.plain_end) == (24, 16, 32)
    lin.bias = None
    assert lin.rows_ref(-1)._obj.bias is None
    lin.ws = None
    assert lin.rows_ref(-1)._obj.ws is None
    lin.w = lin.w[:32]                                   # the same address, fewer rows
    with pytest.raises(ValueError):
        lin.rows_ref(-1)
    lin.d_out, lin.w_scales = 32, lin.w_scales[:32]
    assert lin.rows_ref(-1)._obj.d_out == 32
    other = copy.deepcopy(lin)
    assert other.rows_ref(-1)._obj.w == other.w.data_ptr() != lin.w.data_ptr()


def test_kept_addresses_keep_no_tensor_alive():
    lin = _layer()
    lin.rows_ref(-1)
    gone = []
    weakref.finalize(lin.w, gone.append, 1)
    lin.w = None
    gc.collect()
    assert gone == [1]


@pytest.mark.parametrize("how", range(3))
def test_an_arena_whose_coefficients_move(how):
    a = Z.Arena(torch.zeros(512, dtype=torch.bfloat16), torch.zeros(512), torch.zeros(512))
    first, old, keep = a.coef_ref(-1), a.c.data_ptr(), a.c.detach()
    assert a.coef_ref(-1) is first
    _moves(a.c)[how]()
    d = a.coef_ref(-1)._obj
    assert d.c == a.c.data_ptr() != old and keep is not None and d.k == 512
    a.c = a.c[:200]
    assert a.coef_ref(-1)._obj.k == 200


@pytest.mark.parametrize("how", range(3))
@pytest.mark.parametrize("field", ["pos", "slots", "row_begin", "status"])
def test_a_batch_whose_tensor_moves(field, how):
    i = lambda n: torch.zeros(n, dtype=torch.int32)
    b = Z.CacheBatch(i(4), 2, 8, slots=i(4), row_begin=i(5), status=i(1))
    first = b.ref(-1)
    assert b.ref(-1) is first
    t = getattr(b, field)
    old, keep = t.data_ptr(), t.detach()
    _moves(t)[how]()
    d = b.ref(-1)._obj
    assert getattr(d, field) == t.data_ptr() != old and keep is not None
    b.max_new, b.rows = 3, 9
    assert (b.ref(-1)._obj.max_new, b.ref(-1)._obj.rows) == (3, 9)


def test_a_cache_whose_tensor_moves(monkeypatch):
    monkeypatch.setattr(Z, "_device", lambda t: -1)
    c = Z.Cache.alloc(2, 3, 2, 64, 4, 5, "cpu")
    first = c._ref
    assert c._ref is first
    names = "k v k_scale v_scale table len refs".split()
    for name in names:
        t = getattr(c, name)
        old, keep = t.data_ptr(), t.detach()
        t.data = t.detach().clone()
        d = c._ref._obj
        assert getattr(d, name) == t.data_ptr() != old and keep is not None
        assert [getattr(d, n) for n in names] == [getattr(c, n).data_ptr() for n in names]
    c.k.data = torch.zeros(2, 3, 2, 64, 32, dtype=torch.int8)
    with pytest.raises(ValueError):
        c._ref
