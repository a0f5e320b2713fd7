"""zoact_linear_rows against the plain formula in float64: widths, ranks, epilogues and rows at the ends
of their ranges."""
import copy

import numpy as np
import pytest
import torch

import synth
from paper_2607_01125_amd import zoact as Z

from gpu_helpers import announce, dev, host, t_bf16, t_f32, t_u8

pytestmark = pytest.mark.gpu


def _case(rows, K, N, r, *, flags=0, bias=False, res=False, plain=(0, 0), c_f32=False, seed=0, x_mean=0.0):
    rng = np.random.default_rng([seed, rows, K, N, r])
    q = rng.integers(-7, 8, (N, K))
    packed = ((q[:, ::2] & 15) | ((q[:, 1::2] & 15) << 4)).astype(np.uint8)
    sc = synth.bf16_round((0.007 * np.exp(rng.normal(0, 0.3, (N, K // 128)))).astype(np.float32))
    x = synth.bf16_round((rng.normal(0, 1, (rows, K)) + x_mean).astype(np.float32))
    n_c = N - (plain[1] - plain[0])
    c = rng.normal(0, 0.05, (n_c, r)).astype(np.float32)
    if not c_f32:
        c = synth.bf16_round(c)
    p = synth.bf16_round(rng.normal(0, 1, (rows, r)).astype(np.float32))
    b = synth.bf16_round(rng.normal(0, 0.1, N).astype(np.float32)) if bias else None
    rs = synth.bf16_round(rng.normal(0, 1, (rows, N)).astype(np.float32)) if res else None
    return dict(rows=rows, K=K, N=N, r=r, flags=flags, plain=plain, c_f32=c_f32, q=q, packed=packed, sc=sc, x=x, c=c,
                p=p, b=b, rs=rs)


def _reference(s):
    """y and its error bound before the last rounding, both float64."""
    K, N, rows = s["K"], s["N"], s["rows"]
    w = (s["q"].reshape(N, -1, 128) * s["sc"].astype(np.float64)[:, :, None]).reshape(N, K)
    x = s["x"].astype(np.float64)
    y = x @ w.T
    # magnitudes that enter the fp32 sums: (24 + q) x and the 24 sum x taken out, times the scale
    mag = np.abs(x) @ (np.repeat(s["sc"].astype(np.float64), 128, 1) * 55).T
    if s["r"]:
        cb = synth.bf16_round(s["c"]).astype(np.float64)
        feat = np.r_[0:s["plain"][0], s["plain"][1]:N]
        y[:, feat] += s["p"].astype(np.float64) @ cb.T
        mag[:, feat] += np.abs(s["p"].astype(np.float64)) @ np.abs(cb).T
    if s["b"] is not None:
        y += s["b"].astype(np.float64)
    if s["rs"] is not None:
        y += s["rs"].astype(np.float64)
        mag += np.abs(s["rs"])
    # steps of a sum: 256 products of a group, its scale, the groups of a wave, eight waves, rank, three terms
    steps = 256 + K // 128 + 8 + s["r"] + 4
    tol = steps * 2.0 ** -23 * mag
    if s["flags"] & Z.EPI_RELU:
        y = np.maximum(y, 0)
    if s["flags"] & Z.EPI_SWIGLU:
        f = np.arange(N // 2)
        at = f // 16 * 32 + f % 16
        g, u, tg, tu = y[:, at], y[:, at + 16], tol[:, at], tol[:, at + 16]
        silu = g / (1 + np.exp(-g))
        y = silu * u
        # |silu'| <= 1.1; the exponential, sum, quotient and product round to about 2^-20 together
        tol = 1.1 * tg * (np.abs(u) + tu) + np.abs(silu) * tu + 2.0 ** -20 * np.abs(y)
    return y, tol


def _run(s, f32_out, ws=0):
    lin = Z.Linear(t_u8(s["packed"]), s["K"], s["N"], s["r"], None, 0, t_bf16(s["b"]) if s["b"] is not None else None,
                   t_bf16(s["sc"]), plain=s["plain"])
    if ws:      # (NaN everywhere)
        lin.ws = torch.full((ws,), 255, dtype=torch.uint8, device=dev())
    arena, pad = None, 24
    if s["r"]:
        lin.coef_offset = pad
        c = np.concatenate([np.full(pad, np.nan, np.float32), s["c"].ravel(), np.full(3, np.nan, np.float32)])
        ct = t_f32(c) if s["c_f32"] else t_bf16(c)
        arena = Z.Arena(ct, torch.zeros(1, device=dev()), torch.zeros(1, device=dev()))
    out = s["N"] // 2 if s["flags"] & Z.EPI_SWIGLU else s["N"]
    y = torch.full((s["rows"], out), float("nan"), device=dev(), dtype=torch.float32 if f32_out else torch.bfloat16)
    Z.linear_rows(lin, arena, t_bf16(s["x"]), t_bf16(s["p"]) if s["r"] else None, y,
                  t_bf16(s["rs"]) if s["rs"] is not None else None, s["flags"])
    return y


def _check(s, f32_out, **kw):
    y, tol = _reference(s)
    got = host(_run(s, f32_out, **kw))
    tol = tol + (2.0 ** -24 if f32_out else 2.0 ** -8) * (np.abs(y) + tol)
    bad = ~(np.abs(got - y) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), np.abs(got - y)[bad][:3], tol[bad][:3])


CASES = [
    dict(rows=1, K=128, N=16, r=0),
    dict(rows=1, K=128, N=32, r=1, flags=Z.EPI_SWIGLU),
    dict(rows=1, K=4096, N=256, r=32, res=True),
    dict(rows=2, K=384, N=48, r=5, bias=True),
    dict(rows=5, K=1152, N=80, r=33, flags=Z.EPI_RELU, bias=True, c_f32=True),
    dict(rows=15, K=256, N=96, r=8, flags=Z.EPI_SWIGLU, c_f32=True),
    dict(rows=16, K=512, N=112, r=64, res=True, bias=True),
    dict(rows=17, K=640, N=64, r=256, plain=(16, 40)),
    dict(rows=31, K=2048, N=272, r=16, plain=(0, 100), bias=True),
    dict(rows=33, K=896, N=160, r=100, flags=Z.EPI_SWIGLU, bias=True, res=True),
    dict(rows=48, K=1024, N=1040, r=32, plain=(500, 1040)),
    dict(rows=64, K=1408, N=144, r=7, res=True),
    dict(rows=64, K=128, N=16, r=16, plain=(0, 16)),
    dict(rows=7, K=20480, N=64, r=64, bias=True, res=True),
    dict(rows=3, K=14336, N=128, r=32, res=True, x_mean=2.0),
    dict(rows=1, K=512, N=6144, r=32),
    dict(rows=64, K=256, N=4112, r=32),
    dict(rows=1, K=57472, N=48, r=0),
    dict(rows=16, K=8832, N=32, r=3, flags=Z.EPI_SWIGLU, bias=True),
    dict(rows=4, K=4352, N=8224, r=16, bias=True, res=True),
    dict(rows=12, K=640, N=13344, r=24, flags=Z.EPI_SWIGLU, res=True),
    dict(rows=2, K=8832, N=48, r=40, bias=True),
    dict(rows=10, K=12928, N=160, r=32, flags=Z.EPI_SWIGLU),
    dict(rows=6, K=1024, N=27680, r=8, flags=Z.EPI_SWIGLU),
    dict(rows=3, K=384, N=33040, r=0, res=True),
    dict(rows=20, K=4736, N=352, r=32, flags=Z.EPI_SWIGLU, bias=True),
    dict(rows=13, K=20480, N=320, r=72, bias=True, c_f32=True),
    dict(rows=40, K=4096, N=512, r=32, plain=(100, 300), res=True, c_f32=True),
    dict(rows=9, K=14336, N=96, r=37, flags=Z.EPI_SWIGLU, c_f32=True),
    dict(rows=1, K=14336, N=1040, r=24, plain=(0, 1040), c_f32=True),
    dict(rows=2, K=4096, N=6160, r=16, res=True, c_f32=True),
    dict(rows=24, K=9216, N=160, r=32, bias=True),
    dict(rows=32, K=384, N=8224, r=16, flags=Z.EPI_SWIGLU, c_f32=True),
    dict(rows=29, K=4096, N=4096, r=32, res=True),
    dict(rows=18, K=3200, N=80, r=9, flags=Z.EPI_RELU, bias=True),
]


@pytest.mark.parametrize("f32_out", [False, True])
@pytest.mark.parametrize("kw", CASES, ids=lambda k: f"{k['rows']}x{k['K']}x{k['N']}r{k['r']}")
def test_rows_against_the_formula(kw, f32_out):
    announce("linear_rows", kw, f32_out)
    s = _case(**kw)
    _check(s, f32_out)
    _check(s, f32_out, ws=Z.linear_workspace_bytes())
    _check(s, f32_out, ws=3 * (s["N"] // 16) * 1024)       # room for fewer parts than wanted, or none


@pytest.mark.parametrize("rows,K,N", [(1, 512, 64), (13, 20480, 320), (40, 4096, 512)])
def test_the_residual_may_be_y(rows, K, N):
    announce("in place", rows, K, N)
    s = _case(rows, K, N, 32, res=True)
    want = _run(s, False, ws=Z.linear_workspace_bytes())
    lin = Z.Linear(t_u8(s["packed"]), K, N, 32, w_scales=t_bf16(s["sc"]),
                   ws=torch.empty(Z.linear_workspace_bytes(), dtype=torch.uint8, device=dev()))
    z = torch.zeros(1, device=dev())
    y = t_bf16(s["rs"])
    Z.linear_rows(lin, Z.Arena(t_bf16(s["c"].ravel()), z, z), t_bf16(s["x"]), t_bf16(s["p"]), y, y)
    assert torch.equal(y, want)


def test_codes_and_scales_one_by_one():
    """Rows that are unit vectors read single weights: each of the 16 nibbles' values, at every place of
    a group, comes out as code times scale exactly (fp32 output; the 24 taken out is exact here)."""
    K, N = 256, 32
    q = (np.arange(N)[:, None] + np.arange(K)[None, :]) % 15 - 7
    packed = ((q[:, ::2] & 15) | ((q[:, 1::2] & 15) << 4)).astype(np.uint8)
    sc = synth.bf16_round(np.linspace(0.001, 3.0, N * 2).reshape(N, 2).astype(np.float32))
    lin = Z.Linear(t_u8(packed), K, N, w_scales=t_bf16(sc))
    lin.ws = torch.empty(Z.linear_workspace_bytes(), dtype=torch.uint8, device=dev())
    want = q * np.repeat(sc, 128, 1)
    for k0 in range(0, K, 64):
        x = np.zeros((64, K), np.float32)
        x[np.arange(64), k0 + np.arange(64)] = 1.0
        y = torch.empty(64, N, device=dev())
        announce("linear_rows unit", k0)
        Z.linear_rows(lin, None, t_bf16(x), None, y)
        assert np.array_equal(host(y), want[:, k0:k0 + 64].T.astype(np.float64))


def test_minus_eight_is_read_as_two_complement():
    lin = Z.Linear(t_u8(np.full((16, 64), 0x88)), 128, 16, w_scales=t_bf16(np.ones((16, 1))))
    x = np.zeros((1, 128), np.float32)
    x[0, 77] = 2.0
    y = torch.empty(1, 16, device=dev())
    Z.linear_rows(lin, None, t_bf16(x), None, y)
    assert np.array_equal(host(y), np.full((1, 16), -16.0))


def test_rows_do_not_mix_and_nan_stays_in_its_row():
    s = _case(9, 512, 64, 8, res=True)
    full = host(_run(s, True))
    bad = dict(s, x=s["x"].copy())
    bad["x"][4, 100] = np.nan
    got = host(_run(bad, True))
    assert np.isnan(got[4]).all()
    keep = [i for i in range(9) if i != 4]
    assert np.array_equal(got[keep], full[keep])


def test_same_bits_twice_on_a_side_stream_and_from_a_graph():
    s = _case(13, 1024, 320, 32, bias=True)
    a = _run(s, False)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b = _run(s, False)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(a, b)
    lin = Z.Linear(t_u8(s["packed"]), 1024, 320, 32, None, 0, t_bf16(s["b"]), t_bf16(s["sc"]))
    lin.ws = torch.empty(Z.linear_workspace_bytes(), dtype=torch.uint8, device=dev())
    arena = Z.Arena(t_bf16(s["c"].ravel()), torch.zeros(1, device=dev()), torch.zeros(1, device=dev()))
    x, p = t_bf16(s["x"]), t_bf16(s["p"])
    y, eager = torch.empty_like(a), torch.empty_like(a)
    g = torch.cuda.CUDAGraph()
    Z.linear_rows(lin, arena, x, p, eager)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        Z.linear_rows(lin, arena, x, p, y)
    for i in range(4):
        x.mul_(-0.5)
        Z.linear_rows(lin, arena, x, p, eager)
        y.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i


def test_refusals_on_device_tensors():
    s = _case(4, 256, 32, 8)
    lin = Z.Linear(t_u8(s["packed"]), 256, 32, 0, w_scales=t_bf16(s["sc"]))
    y = torch.empty(4, 32, device=dev(), dtype=torch.bfloat16)
    x = t_bf16(s["x"])
    with pytest.raises(ValueError):
        Z.linear_rows(lin, None, x.t().contiguous().t(), None, y)
    with pytest.raises(ValueError):
        Z.linear_rows(lin, None, x, None, y[:, :16])
    with pytest.raises(ValueError):
        Z.linear_rows(lin, None, x.float(), None, y)
    with pytest.raises(Z.ZoactError):
        Z.linear_rows(Z.Linear(t_bf16(np.zeros((32, 256))), 256, 32), None, x, None, y)
    big = torch.zeros(65, 256, device=dev(), dtype=torch.bfloat16)
    with pytest.raises(Z.ZoactError):
        Z.linear_rows(lin, None, big, None, torch.empty(65, 32, device=dev(), dtype=torch.bfloat16))


def test_a_layer_is_checked_again_after_a_change():
    s, t = _case(2, 256, 32, 8), _case(2, 256, 32, 8, seed=1)
    z = torch.zeros(1, device=dev())
    lin = Z.Linear(t_u8(s["packed"]), 256, 32, 8, w_scales=t_bf16(s["sc"]))
    arena = Z.Arena(t_bf16(s["c"].ravel()), z, z)
    x, p, y = t_bf16(s["x"]), t_bf16(s["p"]), torch.empty(2, 32, dtype=torch.bfloat16, device=dev())
    Z.linear_rows(lin, arena, x, p, y)
    assert torch.equal(y, _run(s, False))
    assert torch.equal(copy.deepcopy(lin).w, lin.w) and torch.equal(copy.deepcopy(arena).c, arena.c)
    lin.w, lin.w_scales, arena.c = t_u8(t["packed"]), t_bf16(t["sc"]), t_bf16(t["c"].ravel())
    Z.linear_rows(lin, arena, t_bf16(t["x"]), t_bf16(t["p"]), y)
    assert torch.equal(y, _run(t, False))
    lin.r = 0
    Z.linear_rows(lin, arena, t_bf16(t["x"]), None, y)
    t["r"] = 0
    assert torch.equal(y, _run(t, False))
    lin.w = lin.w.cpu()
    with pytest.raises(ValueError):
        Z.linear_rows(lin, arena, x, None, y)
    lin.w, lin.r, arena.c = t_u8(t["packed"]), 8, arena.c[:200]
    with pytest.raises(Z.ZoactError):
        Z.linear_rows(lin, arena, x, p, y)


@pytest.mark.parametrize("rows,K,N,flags", [(2, 14336, 96, 0), (13, 20480, 320, Z.EPI_SWIGLU), (50, 4096, 512, Z.EPI_RELU)])
def test_parts_of_the_depth_from_a_graph(rows, K, N, flags):
    """The product and its join, captured once and replayed with eager calls between on a workspace of their own."""
    announce("graph", rows, K, N, flags)
    s = _case(rows, K, N, 40, bias=True, c_f32=True, flags=flags)
    lins = [Z.Linear(t_u8(s["packed"]), K, N, 40, None, 0, t_bf16(s["b"]), t_bf16(s["sc"]),
                     ws=torch.full((Z.linear_workspace_bytes(),), 255, dtype=torch.uint8, device=dev())) for _ in range(2)]
    z = torch.zeros(1, device=dev())
    arena = Z.Arena(t_f32(s["c"].ravel()), z, z)
    x, p = t_bf16(s["x"]), t_bf16(s["p"])
    y, eager = (torch.empty(rows, N // 2 if flags & Z.EPI_SWIGLU else N, dtype=torch.bfloat16, device=dev())
                for _ in range(2))
    Z.linear_rows(lins[0], arena, x, p, y, flags=flags)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        Z.linear_rows(lins[0], arena, x, p, y, flags=flags)
    for i in range(5):
        x.mul_(-0.5)
        Z.linear_rows(lins[1], arena, x, p, eager, flags=flags)
        y.fill_(7.0)
        lins[0].ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i


INF_CASES = [
    dict(rows=1, K=512, N=64, r=8), dict(rows=3, K=1024, N=9216, r=0, flags=Z.EPI_RELU),
    dict(rows=2, K=14336, N=96, r=8, bias=True), dict(rows=13, K=4096, N=64, r=5, res=True),
    dict(rows=9, K=20480, N=320, r=16), dict(rows=20, K=4736, N=352, r=32, bias=True),
    dict(rows=29, K=384, N=8224, r=8), dict(rows=40, K=4096, N=512, r=32, res=True), dict(rows=64, K=1408, N=144, r=7),
]


@pytest.mark.parametrize("kw", INF_CASES, ids=lambda k: f"{k['rows']}x{k['K']}x{k['N']}r{k['r']}")
def test_infinities_are_what_the_formula_says(kw):
    """One infinite x gives its row's features +-inf by the code's sign, and NaN where the code is 0; other rows
    keep their bits."""
    s = _case(**kw)
    row, at = kw["rows"] // 2, 300
    bad = dict(s, x=s["x"].copy())
    bad["x"][row, at] = -np.inf
    for ws in (0, Z.linear_workspace_bytes()):
        announce("infinity", kw, ws)
        full, got = host(_run(s, True, ws=ws)), host(_run(bad, True, ws=ws))
        keep = [i for i in range(kw["rows"]) if i != row]
        assert np.array_equal(got[keep], full[keep])
        with np.errstate(invalid="ignore"):
            want = s["q"][:, at] * -np.inf
        if kw.get("flags"):
            want = np.where(want < 0, 0.0, want)
        assert np.array_equal(got[row], want, equal_nan=True)
    # SwiGLU's two factors: whatever torch makes of the same infinities
    if kw["N"] % 32 == 0 and not kw.get("flags"):
        g = dict(bad, flags=Z.EPI_SWIGLU)
        with np.errstate(invalid="ignore"):
            z = s["q"][:, at] * -np.inf
        f = np.arange(kw["N"] // 2)
        gate, up = (torch.from_numpy(z[f // 16 * 32 + f % 16 + o]) for o in (0, 16))
        got, full = host(_run(g, True)), host(_run(dict(s, flags=Z.EPI_SWIGLU), True))
        assert np.array_equal(got[keep], full[keep])
        assert np.array_equal(got[row], (gate / (1 + torch.exp(-gate)) * up).numpy(), equal_nan=True)


@pytest.mark.parametrize("kw", INF_CASES, ids=lambda k: f"{k['rows']}x{k['K']}x{k['N']}r{k['r']}")
@pytest.mark.parametrize("size", [2.0 ** 121, 2.0 ** 126])
def test_values_near_the_top_overflow_no_earlier_than_the_result(kw, size):
    """x up to 2^127 with scales of 0.007: results of up to 2^125 are finite and within the bound of the sums
    (which grows with x), though 24 x and the sums of codes times x pass fp32's range."""
    s = _case(**dict(kw, flags=0))
    row = kw["rows"] // 2
    s["x"][row] = 0
    s["x"][row, 128:256:9] = size * np.where(np.arange(128, 256, 9) % 2, 1, -1)
    for ws in (0, Z.linear_workspace_bytes()):
        announce("near the top", kw, size, ws)
        y, tol = _reference(s)
        assert np.abs(y).max() < 3e38 and np.abs(y[row]).max() > size * 0.01
        got = host(_run(s, True, ws=ws))
        tol = tol + 2.0 ** -24 * (np.abs(y) + tol)
        assert np.all(np.abs(got - y) <= tol), np.argwhere(~(np.abs(got - y) <= tol))[:3]
