"""The paged 8-bit cache on the GPU: codes and scales bit for bit, pages against a model in Python,
attention against float64 with bounds from its own roundings, and all of them as one step."""
import copy

import numpy as np
import pytest
import torch

import synth
from paper_2607_01125_amd import zoact as Z

import cache_model as cm
from gpu_helpers import announce, dev, host, t_i32

pytestmark = pytest.mark.gpu


class Pair:
    """The cache on the device and its model, driven by the same calls."""

    def __init__(self, n_layers=1, n_pages=24, hkv=2, hd=64, n_slots=6, max_pages=8, garbage=True):
        self.c = Z.Cache.alloc(n_layers, n_pages, hkv, hd, n_slots, max_pages, dev())
        self.m = cm.Model(n_layers, n_pages, hkv, hd, n_slots, max_pages)
        rng = np.random.default_rng(3)
        for t, a in ((self.c.k, self.m.k), (self.c.v, self.m.v)):
            a[...] = rng.integers(-128, 128, a.shape) if garbage else 0
            t.copy_(torch.from_numpy(a))
        for t, a in ((self.c.k_scale, self.m.ks), (self.c.v_scale, self.m.vs)):
            a[...] = np.nan if garbage else 0
            t.copy_(torch.from_numpy(a))
        self.ws = torch.full((Z.cache_workspace_bytes(self.c),), 255, dtype=torch.uint8, device=dev())
        self.status = torch.zeros(1, dtype=torch.int32, device=dev())

    def batch(self, counts, slots=None, max_new=None, ragged=True):
        n = len(counts)
        begin = np.concatenate([[0], np.cumsum(counts)])
        return Z.CacheBatch(torch.full((n,), -7, dtype=torch.int32, device=dev()), max_new or max(max(counts), 1),
                            int(begin[-1]), slots=None if slots is None else t_i32(slots),
                            row_begin=t_i32(begin) if ragged else None, status=self.status)

    def extend(self, counts, slots=None, **kw):
        b = self.batch(counts, slots, **kw)
        announce("extend", str(counts)[:60], str(slots)[:60])
        Z.cache_extend(self.c, b, self.ws)
        pos = self.m.extend(list(range(len(counts))) if slots is None else list(slots), counts)
        assert b.pos.cpu().tolist() == pos
        return b, pos

    def fork(self, src, dst):
        announce("fork", src, dst)
        Z.cache_fork(self.c, t_i32(src), t_i32(dst), self.ws, self.status)
        self.m.fork(src, dst)

    def free(self, slots):
        announce("free", str(slots)[:60])
        Z.cache_free(self.c, t_i32(slots), self.status)
        self.m.free(slots)

    def compact(self):
        announce("compact")
        used = torch.full((1,), -1, dtype=torch.int32, device=dev())
        Z.cache_compact(self.c, self.ws, used)
        assert int(used) == self.m.compact()

    def append(self, layer, k, v, b, pos, counts, slots=None, rope=None):
        """k, v device [rows][hkv * hd]."""
        announce("append", counts, pos)
        Z.cache_append(self.c, layer, k, v, b, rope=rope)
        r = 0
        rp = None if rope is None else tuple(x.cpu().numpy() for x in rope)
        kh, vh = (x.float().cpu().numpy().reshape(-1, self.m.hkv, self.m.hd) for x in (k, v))
        for i, (p, c) in enumerate(zip(pos, counts)):
            if p >= 0 and c:
                self.m.append(layer, i if slots is None else slots[i], p, kh[r:r + c], vh[r:r + c], rp)
            r += c

    def check_pages(self):
        assert np.array_equal(self.c.len.cpu().numpy(), self.m.len)
        assert np.array_equal(self.c.refs.cpu().numpy(), self.m.refs)
        t = self.c.table.cpu().numpy()
        for s in range(len(self.m.len)):
            n = len(self.m.held(s))
            assert np.array_equal(t[s, :n], self.m.table[s, :n]), s
        assert int(self.status) == self.m.status

    def check_codes(self):
        for t, a in ((self.c.k, self.m.k), (self.c.v, self.m.v)):
            g = t.cpu().numpy()
            assert np.array_equal(g, a), (int((g != a).sum()), np.argwhere(g != a)[:4].tolist())
        for t, a in ((self.c.k_scale, self.m.ks), (self.c.v_scale, self.m.vs)):
            assert np.array_equal(t.cpu().numpy(), a, equal_nan=True)


def _rows(rows, width, dtype, seed, std=1.0):
    x = torch.from_numpy(np.random.default_rng(seed).normal(0, std, (rows, width)).astype(np.float32))
    return x.to(dev()).to(dtype)


def _rope(n, hd, theta=1e4):
    a = np.arange(n)[:, None] * theta ** (-2.0 * np.arange(hd // 2) / hd)[None]
    return tuple(torch.from_numpy(f(a).astype(np.float32)).to(dev()) for f in (np.cos, np.sin))


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_append_codes_and_scales_bit_for_bit(hd, dtype, rope):
    """Prompts and single tokens in turn, so that blocks are filled whole, in parts, and grow: every code
    and scale as the header's float32 operations give them, and everything else as it was."""
    pr = Pair(hd=hd, hkv=3, n_pages=20, n_slots=4, max_pages=6)
    rp = _rope(150, hd) if rope else None       # (positions past the table are clamped)
    std = 0.1
    for step, counts in enumerate([[1, 16, 70, 0], [1, 1, 1, 129], [3, 64, 15, 1], [1, 1, 1, 1], [14, 31, 2, 17],
                                   [1, 1, 1, 1]]):
        b, pos = pr.extend(counts)
        wide = _rows(sum(counts), 3 * 3 * hd, dtype, 10 + step, std)
        std *= 1.7                              # later tokens are larger: scales grow
        pr.append(0, wide[:, :3 * hd], wide[:, 6 * hd:], b, pos, counts, rope=rp)
        pr.check_codes()
    pr.check_pages()


def test_append_zero_tiny_and_non_finite_values():
    pr = Pair(hd=32, hkv=1, n_slots=4)
    vals = np.zeros((4, 32), np.float32)
    vals[1] = 1e-45                              # the scale itself underflows to 0
    vals[2] = np.linspace(-1e-38, 1e-38, 32)
    vals[3, 5] = np.inf
    for rows in (vals, np.roll(vals, 1, 0) + 1.0, np.full((4, 32), 2.0, np.float32)):
        counts = [1, 1, 1, 1]
        b, pos = pr.extend(counts)
        t = torch.from_numpy(np.ascontiguousarray(rows, np.float32)).to(dev())
        pr.append(0, t, t, b, pos, counts)
        pr.check_codes()
    bad = torch.full((4, 32), float("nan"), device=dev())
    b, pos = pr.extend([1] * 4)
    pr.append(0, bad, bad, b, pos, [1] * 4)
    pr.check_codes()


@pytest.mark.parametrize("hd", [32, 128])
def test_append_values_next_to_the_middle_between_codes(hd):
    """Quotients k + 1/2, and the numbers beside them, under scales that are powers of two and others."""
    pr = Pair(hd=hd, hkv=1, n_pages=8, n_slots=1, max_pages=8)
    mids = np.arange(-127, 127, dtype=np.float32) + np.float32(0.5)
    up, down = np.nextafter(mids, np.float32(np.inf)), np.nextafter(mids, np.float32(-np.inf))
    for unit in (1.0, 2.0 ** -40, 0.7, 1e-3, 3e30, 2.0 ** -99, 2.0 ** -101, 2.0 ** -126, 2.0 ** -140):
        s = np.float32(127 * unit) * np.float32(1 / 127)
        vals = np.concatenate([mids, up, down]) * s
        vals = np.resize(vals, (-(-vals.size // (hd - 1)), hd - 1))
        rows = np.concatenate([np.full((len(vals), 1), 127 * unit), vals], 1).astype(np.float32)
        rows = np.clip(rows, -np.float32(127 * unit), np.float32(127 * unit))[:48]
        b, pos = pr.extend([len(rows)])
        t = torch.from_numpy(np.ascontiguousarray(rows)).to(dev())
        pr.append(0, t, t, b, pos, [len(rows)])
        pr.check_codes()


def test_append_leaves_out_what_it_cannot_place():
    """pos below 0, a slot or place outside the cache, rows outside the buffers, a page number outside the
    pool: nothing is written for these entries, the others are served."""
    pr = Pair(hd=64, hkv=1, n_slots=5, max_pages=2)
    b, pos = pr.extend([4, 4, 4, 4, 4])
    k = _rows(20, 64, torch.bfloat16, 1)
    b.pos[1] = -1
    b.pos[2] = 2 * 64 - 3
    b.row_begin.copy_(t_i32([0, 4, 8, 12, 16, 21]))
    b.max_new = 5
    pr.c.table[3, 0] = 24
    saved = pr.m.table[3, 0]
    pr.append(0, k, k, b, [0, -1, -1, -1, -1], [4, 4, 4, 4, 4])
    pr.check_codes()
    assert int(pr.status) & Z.STATUS_BAD_ENTRY
    pr.c.table[3, 0] = int(saved)
    b.slots = t_i32([0, 9, -1, 3, 2])
    b.pos.zero_()
    b.row_begin.copy_(t_i32([0, 4, 8, 12, 9, 20]))
    pr.append(0, k, k, b, [0, -1, -1, -1, -1], [4, 4, 4, 4, 4], slots=[0, 0, 0, 0, 0])
    pr.check_codes()


# ------------------------------------------------------------------ pages
@pytest.mark.parametrize("seed", range(6))
def test_pages_against_the_model(seed):
    """Random calls, some of which cannot be served: tables, lengths, counts and contents as the model's."""
    rng = np.random.default_rng(seed)
    pr = Pair(n_layers=2, n_pages=int(rng.integers(9, 40)), hkv=1, hd=32, n_slots=7, max_pages=5)
    for _ in range(40):
        op = rng.choice(["extend", "extend", "extend", "fork", "free", "compact"])
        if op == "extend":
            n = int(rng.integers(1, 8))
            slots = rng.permutation(7)[:n] if rng.random() < 0.8 else rng.integers(-1, 9, n)
            pr.extend([int(x) for x in rng.integers(0, int(rng.choice([2, 30, 130])) + 1, n)], [int(x) for x in slots])
        elif op == "fork":
            n = int(rng.integers(1, 8))
            dst = rng.permutation(7)[:n] if rng.random() < 0.8 else rng.integers(-1, 8, n)
            pr.fork([int(x) for x in rng.integers(0, 7, n)], [int(x) for x in dst])
        elif op == "free":
            pr.free([int(x) for x in rng.integers(-1, 8, int(rng.integers(1, 5)))])
        else:
            pr.compact()
        pr.check_pages()
        pr.check_codes()


def test_fork_permutes_and_copies_on_write():
    pr = Pair(n_pages=30, n_slots=5)
    k = _rows(100 + 30 + 64, 128, torch.bfloat16, 5)
    b, pos = pr.extend([100, 30, 64])
    pr.append(0, k, k, b, pos, [100, 30, 64])
    pr.fork([1, 0, 0, 2, 0], [0, 1, 2, 3, 4])       # slots 0 and 1 change places, 0 is taken three times
    pr.check_pages()
    one = _rows(5, 128, torch.bfloat16, 6)
    b, pos = pr.extend([1] * 5)
    pr.append(0, one, one, b, pos, [1] * 5)
    pr.check_pages()
    pr.check_codes()
    assert len({int(pr.m.table[s, 1]) for s in (1, 2, 4)}) == 3


@pytest.mark.parametrize("n_slots,max_pages", [(40, 2000), (40, 90), (300, 14)])
def test_forks_of_wide_tables_and_many_slots(n_slots, max_pages):
    """Forks that go to one workgroup and to one a slot, of sequences of no page to more than 64."""
    rng = np.random.default_rng(n_slots)
    pr = Pair(n_pages=2500, hkv=1, hd=32, n_slots=n_slots, max_pages=max_pages, garbage=False)
    top = min(max_pages * 64, 5000)
    pr.extend([int(x) for x in rng.integers(0, top + 1, n_slots) * (rng.random(n_slots) < 0.5)])
    for n in (1, 2, 33, n_slots):
        announce("fork", n, n_slots, max_pages)
        pr.fork([int(x) for x in rng.integers(0, n_slots, n)], [int(x) for x in rng.permutation(n_slots)[:n]])
        pr.check_pages()
        pr.fork([int(x) for x in rng.integers(-1, n_slots + 1, n)], [int(x) for x in rng.integers(-1, n_slots + 1, n)])
        pr.check_pages()
        pr.free([int(x) for x in rng.integers(0, n_slots, max(1, n // 8))])
        pr.check_pages()


def test_extend_serves_all_or_nobody():
    pr = Pair(n_pages=4, n_slots=3, max_pages=8)
    pr.extend([64, 65, 0])
    pr.check_pages()
    b, pos = pr.extend([64, 64, 1])
    assert pos == [-1, -1, -1] and pr.m.status == Z.STATUS_NO_PAGES
    pr.check_pages()
    pr.extend([0, 63, 1])
    pr.check_pages()


def test_a_large_pool_and_a_large_batch():
    """The free pages lie behind several thousand used ones; 1024 entries of one token."""
    pr = Pair(n_pages=9001, hkv=1, hd=32, n_slots=1024, max_pages=130, garbage=False)
    pr.extend([130 * 64] * 60)
    pr.extend([1] * 900, [int(x) for x in np.random.default_rng(1).permutation(964)[:900] + 60])
    pr.free(list(range(0, 60, 2)))
    pr.extend([1] * 1024, [int(x) for x in np.random.default_rng(2).permutation(1024)])
    pr.check_pages()
    pr.compact()
    pr.check_pages()


# ------------------------------------------------------------------ attention
def _filled(lens, counts, H, hkv, hd, dtype, rope, n_layers=1, layer=0, seed=0, v_std=1.0):
    n = len(lens)
    mp = max(-(-(L + c) // 64) for L, c in zip(lens, counts)) + 1
    pr = Pair(n_layers=n_layers, n_pages=sum(-(-(L + c) // 64) for L, c in zip(lens, counts)) + 2, hkv=hkv, hd=hd,
              n_slots=n, max_pages=max(mp, 1))
    rp = _rope(max(L + c for L, c in zip(lens, counts)), hd) if rope else None
    for part in (lens, counts):
        if not sum(part):
            b, pos = pr.extend(part)
            continue
        b, pos = pr.extend(part)
        wide = _rows(sum(part), (H + 2 * hkv) * hd, dtype, seed + sum(part))
        pr.append(layer, wide[:, H * hd:(H + hkv) * hd], wide[:, (H + hkv) * hd:] * v_std if v_std != 1.0 else
                  wide[:, (H + hkv) * hd:], b, pos, part, rope=rp)
    pr.check_codes()
    return pr, b, pos, wide[:, :H * hd] if sum(counts) else None, rp


def _check_attention(pr, b, pos, q, counts, H, dtype, rp, max_len, layer=0, split=True, scale=None):
    hkv, hd = pr.m.hkv, pr.m.hd
    scale = np.float32(scale or hd ** -0.5)
    nb = Z.attention_cache_workspace_bytes(pr.c, b, H, max_len)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device=dev()) if split and nb else None
    out = torch.full((b.rows, H * hd), float("nan"), dtype=dtype, device=dev())
    announce("attention", pos, counts, H, hkv, hd, dtype, bool(ws is not None))
    Z.attention_cache(pr.c, layer, q, out, b, H, float(scale), max_len, rope=rp, ws=ws)
    got = host(out).reshape(-1, H, hd)
    qh = host(q).reshape(-1, H, hd)
    rh = None if rp is None else tuple(x.cpu().numpy() for x in rp)
    r = 0
    for i, (p, c) in enumerate(zip(pos, counts)):
        if c:
            k, v = pr.m.values(layer, i, p + c)
            want, mean, mag = cm.attend(qh[r:r + c], k, v, p, float(scale), rh)
            tol = cm.attend_bound(want, mean, mag, p + c, hd, dtype == torch.float32)
            bad = ~(np.abs(got[r:r + c] - want) <= tol)
            assert not bad.any(), (i, int(bad.sum()), np.argwhere(bad)[:3].tolist(),
                                   np.abs(got[r:r + c] - want)[bad][:3], tol[bad][:3])
        r += c
    return out, ws


ATTENTION = [
    # lens, counts, H, hkv, hd
    ([0, 5, 64], [1, 1, 1], 4, 4, 32),
    ([0, 15, 63, 200], [1, 1, 1, 1], 8, 2, 128),
    ([700], [1], 4, 1, 64),
    ([130, 0, 70], [7, 33, 1], 6, 2, 64),
    ([1, 300], [20, 5], 40, 2, 32),
    ([64, 128], [64, 65], 2, 2, 128),
    ([10], [1], 33, 1, 128),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("lens,counts,H,hkv,hd", ATTENTION)
def test_attention_against_float64(lens, counts, H, hkv, hd, rope, dtype):
    pr, b, pos, q, rp = _filled(lens, counts, H, hkv, hd, dtype, rope)
    n = max(L + c for L, c in zip(lens, counts))
    whole, _ = _check_attention(pr, b, pos, q, counts, H, dtype, rp, n, split=False)
    _check_attention(pr, b, pos, q, counts, H, dtype, rp, n)
    # a bound that is too small or far too large only shapes the work
    _check_attention(pr, b, pos, q, counts, H, dtype, rp, 1)
    _check_attention(pr, b, pos, q, counts, H, dtype, rp, 100000)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_of_a_long_sequence_in_many_splits(dtype):
    """5000 tokens of one sequence: splits of several pages, the last one short; the second layer."""
    pr, b, pos, q, rp = _filled([4999], [1], 8, 2, 64, dtype, True, n_layers=2, layer=1)
    _check_attention(pr, b, pos, q, [1], 8, dtype, rp, 5000, layer=1)
    out, ws = _check_attention(pr, b, pos, q, [1], 8, dtype, rp, 5000, layer=1)
    assert ws is not None
    again = torch.empty_like(out)
    Z.attention_cache(pr.c, 1, q, again, b, 8, float(np.float32(64 ** -0.5)), 5000, rope=rp, ws=ws)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [-0.4, 0.4])
@pytest.mark.parametrize("lens,counts", [([40, 130, 16], [1, 1, 2]), ([40, 0, 150], [40, 70, 20])])
def test_attention_blocks_of_zero_keys_and_a_negative_scale(lens, counts, scale, dtype):
    """Blocks whose keys are all zero have scale 0: their scores are 0, neither masked nor NaN, also where the
    row's own end lies in one."""
    H, hkv, hd = 4, 2, 64
    pr = Pair(n_pages=16, hkv=hkv, hd=hd, n_slots=3, max_pages=4)
    for part in (lens, counts):
        b, pos = pr.extend(part)
        x = _rows(sum(part), (H + 2 * hkv) * hd, dtype, 7 + sum(part))
        keys = x[:, H * hd:(H + hkv) * hd]
        at = torch.cat([torch.arange(p, p + c) for p, c in zip(pos, part)]).to(dev())
        keys[(at < 16) | ((at >= 32) & (at < 48)) | (at >= 112)] = 0
        pr.append(0, keys, x[:, (H + hkv) * hd:], b, pos, part)
    pr.check_codes()
    for split in (False, True):
        _check_attention(pr, b, pos, x[:, :H * hd], counts, H, dtype, None, 220, split=split, scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [1e2, 1e4, 1e8])
@pytest.mark.parametrize("lens,counts", [([300, 64], [1, 1]), ([130, 1], [40, 70])])
def test_attention_of_very_large_scores_takes_the_largest(lens, counts, size, dtype):
    """Scores of up to 2^60, whose rounding alone passes the exponential's range: each row is the value of
    its largest score (rows whose two largest are closer than their rounding left out)."""
    H, hkv, hd = 4, 2, 64
    pr, b, pos, q, _ = _filled(lens, counts, H, hkv, hd, dtype, False)
    pr.c.k_scale.mul_(size)
    pr.m.ks *= np.float32(size)
    big = (q.float() * size).to(dtype)
    qh = host(big).reshape(-1, H, hd)
    for ws in (None, torch.empty(Z.attention_cache_workspace_bytes(pr.c, b, H, 400), dtype=torch.uint8, device=dev())):
        out = torch.empty(b.rows, H * hd, dtype=dtype, device=dev())
        Z.attention_cache(pr.c, 0, big, out, b, H, 0.125, 400, ws=ws)
        got, r, seen = host(out).reshape(-1, H, hd), 0, 0
        for i, (p, c) in enumerate(zip(pos, counts)):
            k, v = pr.m.values(0, i, p + c)
            for j in range(c):
                for h in range(H):
                    kk, vv = (x[:p + j + 1, h // (H // hkv)].astype(np.float64) for x in (k, v))
                    sc = kk @ qh[r + j, h] * 0.125
                    top = np.argsort(sc)[::-1][:2]
                    err = 2.0 ** -10 * 0.125 * float(np.abs(kk).max(0) @ np.abs(qh[r + j, h]))
                    if len(top) > 1 and sc[top[0]] - sc[top[1]] < err + 60:
                        continue
                    seen += 1
                    want = vv[top[0]]
                    assert np.all(np.abs(got[r + j, h] - want) <= 2.0 ** -7 * np.abs(want) + 1e-12), (i, j, h)
            r += c
        assert seen >= b.rows * H // 3


def test_attention_sharp_and_flat_scores():
    """A scale that makes the softmax nearly a choice, and one that makes it nearly a mean."""
    pr, b, pos, q, rp = _filled([400, 90], [1, 3], 4, 2, 64, torch.float32, False)
    for scale in (1.0, 2.0, 1e-4):
        _check_attention(pr, b, pos, q, [1, 3], 4, torch.float32, rp, 403, scale=scale)


def test_attention_rows_without_a_place_are_zero_and_others_untouched():
    pr, b, pos, q, rp = _filled([70, 20, 5], [2, 2, 2], 4, 2, 64, torch.bfloat16, False)
    ok = _check_attention(pr, b, pos, q, [2, 2, 2], 4, torch.bfloat16, rp, 72)[0]
    b.pos[1] = -1
    big = torch.full((9, 256), 3.0, dtype=torch.bfloat16, device=dev())
    qq = torch.cat([q, q[:3]])
    b.rows = 9
    for max_len in (72, 4096):
        ws = torch.empty(max(16, Z.attention_cache_workspace_bytes(pr.c, b, 4, max_len)), dtype=torch.uint8, device=dev())
        big.fill_(3.0)
        Z.attention_cache(pr.c, 0, qq, big, b, 4, 0.125, max_len, ws=ws)
        assert torch.equal(big[:2], ok[:2]) and torch.equal(big[4:6], ok[4:6])
        assert (big[2:4] == 0).all() and (big[6:] == 3).all()
    # a slot that is none, and a range of rows that is none
    b.pos[1] = 20
    b.slots = t_i32([0, 3, 2])
    big.fill_(3.0)
    Z.attention_cache(pr.c, 0, qq, big, b, 4, 0.125, 72)
    assert (big[2:4] == 0).all() and torch.equal(big[4:6], ok[4:6])
    assert int(pr.status) & Z.STATUS_BAD_ENTRY
    b.slots = None
    b.row_begin.copy_(t_i32([0, 2, 4, 10]))
    big.fill_(3.0)
    Z.attention_cache(pr.c, 0, qq, big, b, 4, 0.125, 72)
    assert torch.equal(big[:4], ok[:4]) and (big[4:] == 3).all()


def test_attention_skips_a_page_that_is_none():
    pr, b, pos, q, rp = _filled([130], [1], 2, 1, 32, torch.float32, False)
    page = int(pr.c.table[0, 1])
    for bad in (-1, int(pr.c.refs.numel()), 2 ** 31 - 1):
        pr.c.table[0, 1] = bad
        pr.status.zero_()
        out = torch.empty(1, 64, device=dev())
        announce("bad page", bad)
        Z.attention_cache(pr.c, 0, q, out, b, 2, 0.2, 131)
        assert int(pr.status) == Z.STATUS_BAD_ENTRY
        k, v = pr.m.values(0, 0, 131)
        keep = np.r_[0:64, 128:131]
        want, mean, mag = cm.attend(host(q).reshape(1, 2, 32), k[keep], v[keep], len(keep) - 1, float(np.float32(0.2)))
        assert (np.abs(host(out).reshape(1, 2, 32) - want) <= cm.attend_bound(want, mean, mag, 131, 32, True)).all()
    pr.c.table[0, 1] = page


def test_a_value_that_is_not_finite_reaches_those_who_see_it():
    """NaN in one block of one head: rows that see the block give NaN there, earlier rows and other heads
    do not; NaN in q stays in its row and head."""
    pr = Pair(hkv=2, hd=32, n_slots=2)
    counts = [40, 40]
    b, pos = pr.extend(counts)
    w = _rows(80, 64 + 128, torch.float32, 4)
    q, k, v = w[:, :64].contiguous(), w[:, 64:128].clone(), w[:, 128:].clone()
    k[35, 40] = float("inf")                        # entry 0, token 35 (block 2), head 1
    v[40 + 20, 3] = float("nan")                    # entry 1, token 20 (block 1), head 0
    pr.append(0, k, v, b, pos, counts)
    pr.check_codes()
    q[10, 5] = float("nan")                         # entry 0, row 10, head 0
    out = torch.empty(80, 64, device=dev())
    Z.attention_cache(pr.c, 0, q, out, b, 2, 0.2, 40)
    o = host(out).reshape(2, 40, 2, 32)
    want = np.zeros((2, 40, 2), bool)
    want[0, 32:, 1] = True
    want[1, 16:, 0] = True
    want[0, 10, 0] = True
    # (a block's scale is one: a row that ends inside the block sees it)
    assert np.array_equal(np.isnan(o).all(-1), want) and np.array_equal(np.isnan(o).any(-1), want)


# ------------------------------------------------------------------ together
def test_a_step_captured_and_replayed():
    """extend, append and attention as one graph, replayed on growing sequences with eager work between:
    every replay as the eager calls on a second cache."""
    H, hkv, hd, n = 4, 2, 64, 3
    a, e = Pair(n_pages=30, n_slots=n), Pair(n_pages=30, n_slots=n)
    rp = _rope(600, hd)
    first = _rows(60 + 1 + 120, 2 * hkv * hd, torch.bfloat16, 1)
    for pr in (a, e):
        b, pos = pr.extend([60, 1, 120])
        pr.append(0, first[:, :hkv * hd], first[:, hkv * hd:], b, pos, [60, 1, 120], rope=rp)
    x = _rows(n, (H + 2 * hkv) * hd, torch.bfloat16, 2)
    q, k, v = x[:, :H * hd], x[:, H * hd:(H + hkv) * hd], x[:, (H + hkv) * hd:]
    outs = [torch.empty(n, H * hd, dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    bs = [pr.batch([1] * n, ragged=False) for pr in (a, e)]
    nb = Z.attention_cache_workspace_bytes(a.c, bs[0], H, 512)
    wss = [torch.empty(max(nb, 16), dtype=torch.uint8, device=dev()) for _ in range(2)]

    def step(i, pr):
        Z.cache_extend(pr.c, bs[i], pr.ws)
        Z.cache_append(pr.c, 0, k, v, bs[i], rope=rp)
        Z.attention_cache(pr.c, 0, q, outs[i], bs[i], H, 0.125, 512, rope=rp, ws=wss[i])

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step(0, a)
    for i in range(10):
        x.copy_(_rows(n, (H + 2 * hkv) * hd, torch.bfloat16, 50 + i))
        g.replay()
        torch.cuda.synchronize()
        step(1, e)
        assert torch.equal(outs[0], outs[1]), i
        assert torch.equal(a.c.len, e.c.len) and torch.equal(a.c.refs, e.c.refs)
        if i == 4:
            for pr in (a, e):
                Z.cache_fork(pr.c, t_i32([2]), t_i32([0]), pr.ws)
    assert int(a.c.len[0]) == 120 + 10 and int(a.status) == 0


def test_bounds_far_past_the_table():
    """max_new and max_len are bounds only: large ones give what the exact ones give."""
    outs = []
    for far in (False, True):
        pr = Pair(n_pages=12, n_slots=2, hkv=2, hd=64, max_pages=6, garbage=False)
        x = _rows(230, 3 * 128, torch.bfloat16, 4)
        for lens in ([100, 130], [1, 60]):
            rows = sum(lens)
            b = pr.batch(lens, max_new=2 ** 31 - 1 if far else None)
            announce("bounds", far, lens)
            Z.cache_extend(pr.c, b, pr.ws)
            Z.cache_append(pr.c, 0, x[:rows, 128:256], x[:rows, 256:], b)
        b.max_new = 2 ** 17 if far else 60
        out = torch.empty(61, 128, dtype=torch.bfloat16, device=dev())
        Z.attention_cache(pr.c, 0, x[:61, :128], out, b, 2, 0.1, 2 ** 63 - 1 if far else 190)
        outs.append((out.float(), pr.c.table, pr.c.len, b.pos))
    for a, b in zip(outs[0][1:], outs[1][1:]):
        assert torch.equal(a, b)
    # both within a rounding of the probabilities (2^-12) and of bf16 (2^-8) of means of values
    assert float((outs[0][0] - outs[1][0]).abs().max()) <= 2 * (2.0 ** -12 + 2.0 ** -8) * float(x.float().abs().max())


def test_a_batch_of_no_rows():
    pr = Pair(n_pages=4, n_slots=3)
    b = pr.batch([0, 0])
    none = torch.empty(0, 128, dtype=torch.bfloat16, device=dev())
    Z.cache_extend(pr.c, b, pr.ws)
    Z.cache_append(pr.c, 0, none, none, b)
    Z.attention_cache(pr.c, 0, none, torch.empty_like(none), b, 2, 1.0, 1)
    assert b.pos.tolist() == [0, 0] and pr.c.len.tolist() == [0, 0, 0]


def test_a_batch_is_checked_again_after_a_change():
    pr = Pair()
    b, _ = pr.extend([1, 1])
    b.slots = torch.zeros(2, dtype=torch.int64, device=dev())
    with pytest.raises(ValueError):
        Z.cache_extend(pr.c, b, pr.ws)
    b.slots = t_i32([1, 0])
    Z.cache_extend(pr.c, b, pr.ws)
    assert pr.c.len.tolist()[:2] == [2, 2]


def test_copies_are_caches_and_batches_of_their_own():
    pr = Pair()
    b, _ = pr.extend([3, 70])
    c2, b2 = copy.deepcopy(pr.c), copy.deepcopy(b)
    assert (c2.index, c2.n_kv_heads, c2.head_dim) == (pr.c.index, pr.c.n_kv_heads, pr.c.head_dim)
    Z.cache_extend(c2, b2, pr.ws)
    assert c2.len.tolist()[:2] == [6, 140] and pr.c.len.tolist()[:2] == [3, 70]
    assert b2.pos.tolist() == [3, 70] and b.pos.tolist() == [0, 0]
    pr.check_pages()


def test_two_streams_with_their_own_caches():
    """The same work on two streams at once, each with its cache and workspaces, gives the same bits."""
    res = []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    prs = [Pair(n_pages=40, n_slots=2, hkv=2, hd=128) for _ in streams]
    x = _rows(2 * 300, 3 * 256, torch.bfloat16, 9)
    torch.cuda.synchronize()
    for st, pr in zip(streams, prs):
        with torch.cuda.stream(st):
            b = pr.batch([300, 300])
            out = torch.empty(600, 256, dtype=torch.bfloat16, device=dev())
            Z.cache_extend(pr.c, b, pr.ws)
            Z.cache_append(pr.c, 0, x[:, 256:512], x[:, 512:], b)
            Z.attention_cache(pr.c, 0, x[:, :256], out, b, 2, 0.1, 300)
            res.append(out)
    torch.cuda.synchronize()
    assert torch.equal(res[0], res[1]) and torch.isfinite(res[0].float()).all()


def test_refusals_on_device_tensors():
    pr = Pair()
    b, _ = pr.extend([1, 1])
    k = _rows(2, 128, torch.bfloat16, 0)
    with pytest.raises(ValueError):
        Z.cache_append(pr.c, 0, k[:, :64], k, b)
    with pytest.raises(ValueError):
        Z.cache_append(pr.c, 0, k.half(), k.half(), b)
    with pytest.raises(Z.ZoactError):
        Z.cache_append(pr.c, 1, k, k, b)
    with pytest.raises(ValueError):
        Z.attention_cache(pr.c, 0, k, k.float(), b, 2, 1.0, 5)
    with pytest.raises(Z.ZoactError):
        Z.attention_cache(pr.c, 0, k[:, :64], torch.empty(2, 64, dtype=torch.bfloat16, device=dev()), b, 1, 1.0, 5)
    with pytest.raises(Z.ZoactError):
        Z.cache_extend(pr.c, b, pr.ws[:64])
    with pytest.raises(ValueError):
        Z.cache_extend(pr.c, b, pr.ws.cpu())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_many_chunks_at_once(hd, dtype):
    """Enough chunks of rows that workgroups take 128 columns each (bf16), ragged, behind lengths that end
    anywhere in a page; three of the entries against float64, one of no rows."""
    rng = np.random.default_rng(hd)
    n, H, hkv = 40, 32, 8
    lens = [int(x) for x in rng.integers(0, 100, n)]
    counts = [int(x) for x in rng.integers(60, 131, n)]
    counts[3], counts[7], lens[9] = 130, 0, 64
    c = Z.Cache.alloc(1, sum(-(-(a + b) // 64) for a, b in zip(lens, counts)), hkv, hd, n, 4, dev())
    ws = torch.empty(Z.cache_workspace_bytes(c), dtype=torch.uint8, device=dev())
    rp = _rope(240, hd)
    for part in (lens, counts):
        begin = np.concatenate([[0], np.cumsum(part)])
        b = Z.CacheBatch(torch.empty(n, dtype=torch.int32, device=dev()), max(part), int(begin[-1]),
                         row_begin=t_i32(begin), status=torch.zeros(1, dtype=torch.int32, device=dev()))
        Z.cache_extend(c, b, ws)
        x = _rows(int(begin[-1]), (H + 2 * hkv) * hd, dtype, sum(part))
        Z.cache_append(c, 0, x[:, H * hd:(H + hkv) * hd], x[:, (H + hkv) * hd:], b, rope=rp)
    out = torch.full((b.rows, H * hd), float("nan"), dtype=dtype, device=dev())
    announce("many chunks", hd, dtype)
    Z.attention_cache(c, 0, x[:, :H * hd], out, b, H, hd ** -0.5, 240, rope=rp)
    assert torch.isfinite(out).all() and int(b.status) == 0 and b.pos.tolist() == lens
    m = cm.Model(1, c.refs.numel(), hkv, hd, n, 4)
    for a, t in ((m.k, c.k), (m.v, c.v), (m.ks, c.k_scale), (m.vs, c.v_scale), (m.table, c.table)):
        a[...] = t.cpu().numpy()
    rh = tuple(t.cpu().numpy() for t in rp)
    for i in (3, 9, n - 1):
        r0, r1, L = int(begin[i]), int(begin[i + 1]), lens[i]
        k, v = m.values(0, i, L + counts[i])
        want, mean, mag = cm.attend(host(x[r0:r1, :H * hd]).reshape(-1, H, hd), k, v, L, float(np.float32(hd ** -0.5)), rh)
        tol = cm.attend_bound(want, mean, mag, L + counts[i], hd, dtype == torch.float32)
        bad = ~(np.abs(host(out[r0:r1]).reshape(-1, H, hd) - want) <= tol)
        assert not bad.any(), (i, int(bad.sum()), np.argwhere(bad)[:3].tolist())


def test_pools_past_two_gigabytes():
    """Pages and layers whose bytes lie past 2^31: the same values as in a small pool."""
    hkv, hd, H, big_pages = 1, 128, 4, 150_000
    small = Z.Cache.alloc(1, 12, hkv, hd, 2, 8, dev())
    big = Z.Cache.alloc(3, big_pages, hkv, hd, 2, 8, dev())
    big.refs[:big_pages - 9] = 1                    # the free ones are the last
    outs = []
    x = _rows(300 + 131, (H + 2 * hkv) * hd, torch.bfloat16, 3)
    for c, layer in ((small, 0), (big, 2)):
        ws = torch.empty(Z.cache_workspace_bytes(c), dtype=torch.uint8, device=dev())
        st = torch.zeros(1, dtype=torch.int32, device=dev())
        b = Z.CacheBatch(torch.empty(2, dtype=torch.int32, device=dev()), 300, 431, row_begin=t_i32([0, 300, 431]),
                         status=st)
        announce("large pool", c.refs.numel(), layer)
        Z.cache_extend(c, b, ws)
        Z.cache_append(c, layer, x[:, H * hd:(H + hkv) * hd], x[:, (H + hkv) * hd:], b)
        out = torch.empty(431, H * hd, dtype=torch.bfloat16, device=dev())
        Z.attention_cache(c, layer, x[:, :H * hd], out, b, H, 0.1, 300)
        assert int(st) == 0
        # one token more of a forked sequence: the copy of its last page lies far out too
        Z.cache_free(c, t_i32([1]), st)
        Z.cache_fork(c, t_i32([0]), t_i32([1]), ws, st)
        one = Z.CacheBatch(torch.empty(2, dtype=torch.int32, device=dev()), 1, 2, status=st)
        Z.cache_extend(c, one, ws)
        Z.cache_append(c, layer, x[:2, H * hd:(H + hkv) * hd], x[:2, (H + hkv) * hd:], one)
        last = torch.empty(2, H * hd, dtype=torch.bfloat16, device=dev())
        Z.attention_cache(c, layer, x[:2, :H * hd], last, one, H, 0.1, 301)
        assert int(st) == 0
        outs.append((out, last, c.table.cpu() - (big_pages - 9 if c is big else 0)))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert int(outs[1][2][0, :5].min()) >= 0
    big.refs[:big_pages - 9] = 0
    used = torch.empty(1, dtype=torch.int32, device=dev())
    Z.cache_compact(big, torch.empty(Z.cache_workspace_bytes(big), dtype=torch.uint8, device=dev()), used)
    assert int(used) == int((big.refs > 0).sum()) and int(big.table[:, :5].max()) < int(used)
    again = torch.empty(2, H * hd, dtype=torch.bfloat16, device=dev())
    Z.attention_cache(big, 2, x[:2, :H * hd], again, one, H, 0.1, 301)
    assert torch.equal(again, outs[1][1])


# ------------------------------------------------------------------ value scales that differ between blocks
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("larger", [2.0 ** 20, 2.0 ** 45])
@pytest.mark.parametrize("lens,counts,H,hkv", [([10], [12], 1, 1), ([0, 60], [40, 50], 4, 2), ([14, 47], [4, 4], 8, 2)])
def test_rows_do_not_see_the_scales_of_later_values(lens, counts, H, hkv, larger, dtype):
    """New rows of one page, the values of its later blocks 2^20 and 2^45 times larger: a row that sees only the
    earlier blocks keeps the precision it has alone.  (A probability times its value scale is a number of f16 whose
    unit puts the row's largest scale below 2^14, so it is off by 2^-25 of that unit at most beside its relative error:
    2^-38 of the largest scale the row sees, 127 times that in the result for each token.)"""
    hd = 64
    pr = Pair(hkv=hkv, hd=hd, n_slots=len(lens), max_pages=3)
    for part in (lens, counts):
        b, pos = pr.extend(part)
        x = _rows(sum(part), (H + 2 * hkv) * hd, dtype, 21 + sum(part))
        v = x[:, (H + hkv) * hd:]
        at = torch.cat([torch.arange(p, p + c) for p, c in zip(pos, part)]).to(dev())
        # (in the second half of the new rows' blocks)
        from_ = [L + c // 2 if part is counts else 10 ** 6 for L, c in zip(lens, counts)]
        first = torch.repeat_interleave(torch.tensor(from_), torch.tensor(part)).to(dev())
        big = at // 16 >= first // 16
        v[big] *= larger
        seen = (~big).cpu().numpy()
        pr.append(0, x[:, H * hd:(H + hkv) * hd], v, b, pos, part)
    pr.check_codes()
    assert seen.any() and not seen.all()
    scale, out = float(np.float32(hd ** -0.5)), torch.empty(sum(counts), H * hd, dtype=dtype, device=dev())
    announce("later scales", pos, counts, H, hkv, larger, dtype)
    Z.attention_cache(pr.c, 0, x[:, :H * hd], out, b, H, scale, 128)
    r = 0
    for i, (p, c) in enumerate(zip(pos, counts)):
        k, v = pr.m.values(0, i, p + c)
        want, mean, mag = cm.attend(host(x[r:r + c, :H * hd]).reshape(c, H, hd), k, v, p, scale)
        tol = cm.attend_bound(want, mean, mag, p + c, hd, dtype == torch.float32)
        vs = np.concatenate([pr.m.vs[0, page].T for page in pr.m.held(i)]).max(1)        # [blocks], of all heads
        top = np.array([vs[:t // 16 + 1].max() for t in range(p, p + c)])
        tol += (np.arange(p, p + c) + 1)[:, None, None] * 127 * 2.0 ** -38 * top[:, None, None]
        bad = ~(np.abs(host(out[r:r + c]).reshape(c, H, hd) - want) <= tol)
        assert not bad.any(), (i, int(bad.sum()), np.argwhere(bad)[:3].tolist())
        r += c
    # the small rows against the same rows of a cache that ends before the large ones
    alone = [int(s.sum()) for s in np.split(seen, np.cumsum(counts)[:-1])]
    begin = t_i32(np.concatenate([[0], np.cumsum(alone)]))
    few = Z.CacheBatch(t_i32(pos), max(counts), sum(alone), row_begin=begin)
    keep = torch.from_numpy(np.flatnonzero(seen)).to(dev())
    got = torch.empty(sum(alone), H * hd, dtype=dtype, device=dev())
    Z.attention_cache(pr.c, 0, x[keep][:, :H * hd].contiguous(), got, few, H, scale, 128)
    assert torch.equal(out[keep], got)


def _pages_f64(c, slots, n_pages):
    """Keys and values [slots][tokens][hkv][hd] of the first pages of a layer's slots, dequantised, float64."""
    t = c.table[:slots, :n_pages].long()
    hkv, hd = c.n_kv_heads, c.head_dim
    k = c.k[0][t].double() * c.k_scale[0][t].double().repeat_interleave(16, -1)[..., None]     # [s][p][h][64][d]
    place = torch.tensor([cm.v_place(i) for i in range(64)], device=dev())
    v = c.v[0][t][..., place].double() * c.v_scale[0][t].double().repeat_interleave(16, -1)[..., None, :]
    return (k.permute(0, 1, 3, 2, 4).reshape(slots, -1, hkv, hd), v.permute(0, 1, 4, 2, 3).reshape(slots, -1, hkv, hd))


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("slots,count", [(512, 1), (64, 8)])
def test_fp32_rows_of_few_weighty_tokens_keep_their_bits(slots, count, hd):
    """Rows whose weight lies on six tokens (two blocks of a whole page and of a partial one, the rest e^-80 below),
    in both tile forms: where a term of p vsc is cut wrongly it shows, for 2^-11 of it is lost.  The bound is the
    usual one over those six."""
    H, hkv, L = 32, 8, 96
    sel = [5, 22, 39, 60, 70, 90]
    pr = Pair(n_pages=3 * slots, hkv=hkv, hd=hd, n_slots=slots, max_pages=3, garbage=False)
    rng = torch.Generator(device="cuda").manual_seed(hd + count)
    for n in (L, count):
        b = pr.batch([n] * slots)
        Z.cache_extend(pr.c, b, pr.ws)
        kv = torch.randn(2, slots * n, hkv, hd, generator=rng, device=dev()) * 0.2
        kv[0, :, :, 0] = -1.0
        if n == L:
            kv[0].view(slots, n, hkv, hd)[:, sel, :, 0] = 0.0
        Z.cache_append(pr.c, 0, kv[0].view(-1, hkv * hd), kv[1].view(-1, hkv * hd), b)
    q = torch.randn(slots * count, H, hd, generator=rng, device=dev())
    q[:, :, 0] = 640.0
    scale = 0.125
    out = torch.empty(slots * count, H * hd, device=dev())
    announce("few tokens", slots, count, hd)
    Z.attention_cache(pr.c, 0, q.view(-1, H * hd), out, b, H, scale, L + count)
    k, v = (x[:, sel].repeat_interleave(H // hkv, 2) for x in _pages_f64(pr.c, slots, 2))      # [s][6][H][d]
    q64 = q.double().view(slots, count, 1, H, hd)
    w = ((q64 * k[:, None]).sum(-1) * scale).softmax(2)[..., None]                             # [s][c][6][H][1]
    want, mean = ((w * x[:, None]).sum(2) for x in (v, v.abs()))
    mag = ((q64.abs() * k[:, None].abs()).sum(-1) * scale).amax(2)[..., None]
    tol = cm.attend_bound(want.cpu().numpy(), mean.cpu().numpy(), mag.cpu().numpy(), len(sel), hd, True)
    bad = ~(np.abs(host(out).reshape(want.shape) - want.cpu().numpy()) <= tol)
    assert not bad.any(), (int(bad.any(-1).sum()), np.argwhere(bad)[:3].tolist())


# ------------------------------------------------------------------ splits
@pytest.mark.parametrize("lens,count,H", [([2000, 70], 1, 2), ([6000, 9], 1, 1), ([2000, 70], 20, 2), ([9000, 1], 1, 20)])
def test_a_value_that_is_not_finite_reaches_those_who_see_it_through_splits(lens, count, H):
    """A NaN value 130 nats below the row's largest score, in another split (few-split and wide joins, both
    tile forms): the row gives NaN, as without a workspace; a row that does not see it does not."""
    hd, n = 32, len(lens)
    pr = Pair(n_pages=sum(-(-(L + count) // 64) for L in lens), hkv=1, hd=hd, n_slots=n, max_pages=-(-max(lens) // 64) + 1,
              garbage=False)
    counts = [count] * n
    for part in (lens, counts):
        b = pr.batch(part)
        Z.cache_extend(pr.c, b, pr.ws)
        rows = sum(part)
        k, v = torch.zeros(rows, hd, device=dev()), _rows(rows, hd, torch.float32, 8)
        k[:, 0] = 1.0
        if part is lens:
            k[:lens[0] // 2, 0] = -1.0             # entry 0: far below the rest, in its first half
            v[100, 5] = float("nan")
        Z.cache_append(pr.c, 0, k, v, b)
    q = torch.zeros(sum(counts), H * hd, device=dev())
    q[:, ::hd] = 65.0
    outs = []
    nb = Z.attention_cache_workspace_bytes(pr.c, b, H, max(lens) + count)
    assert nb > 0
    for ws in (None, torch.full((nb,), 255, dtype=torch.uint8, device=dev())):
        out = torch.zeros(sum(counts), H * hd, device=dev())
        announce("nan in a split", lens, count, H, ws is not None)
        Z.attention_cache(pr.c, 0, q, out, b, H, 1.0, max(lens) + count, ws=ws)
        o = host(out).reshape(n, count, H, hd)
        assert np.isnan(o[0]).all() and np.isfinite(o[1]).all()
        outs.append(np.isnan(o))
    assert np.array_equal(*outs)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,counts,H,hkv,hd", [
    ([1500, 30, 700], [70, 40, 65], 4, 2, 64),        # chunks in up to eight splits, some of them empty
    ([2300, 5], [17, 33], 2, 1, 128),
    ([9000, 40, 2], [1, 1, 1], 20, 1, 32),            # a tile of more than 16 columns and more than eight splits
    ([5000, 600], [9, 3], 6, 2, 64),
])
def test_chunks_behind_long_prompts_in_splits(lens, counts, H, hkv, hd, dtype):
    """The 64-column form with partial results: against float64, the same on every run, and with an entry that has no
    place between the others."""
    pr, b, pos, q, rp = _filled(lens, counts, H, hkv, hd, dtype, True)
    n = max(L + c for L, c in zip(lens, counts))
    out, ws = _check_attention(pr, b, pos, q, counts, H, dtype, rp, n)
    assert ws is not None and max(counts) * (H // hkv) > 16
    again = torch.full_like(out, 3.0)
    scale = float(np.float32(hd ** -0.5))
    ws.fill_(255)
    Z.attention_cache(pr.c, 0, q, again, b, H, scale, n, rope=rp, ws=ws)
    assert torch.equal(out, again)
    b.pos[1] = -1
    ws.fill_(255)
    Z.attention_cache(pr.c, 0, q, again, b, H, scale, n, rope=rp, ws=ws)
    r0, r1 = counts[0], counts[0] + counts[1]
    assert torch.equal(again[:r0], out[:r0]) and torch.equal(again[r1:], out[r1:]) and (again[r0:r1] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,counts,H,hkv,hd", [([5, 300], [1, 1], 4, 2, 64), ([40, 200], [30, 9], 4, 2, 128),
                                                  ([3000], [1], 2, 1, 32), ([5000], [2], 2, 1, 64), ([1500], [40], 2, 1, 32)])
def test_values_near_the_top_of_the_range(lens, counts, H, hkv, hd, dtype):
    """Values of about 2^126: their weighted sums pass fp32's range, their means do not (unsplit, in few and in many
    splits, both tile forms)."""
    pr, b, pos, q, rp = _filled(lens, counts, H, hkv, hd, dtype, False)
    factor = 2.0 ** 126 / float(pr.c.v_scale[0, pr.c.table[0, 0].long(), 0, 0] * 127)
    pr.c.v_scale.mul_(factor)
    pr.m.vs *= np.float32(factor)
    n = max(L + c for L, c in zip(lens, counts))
    for split in (False, True):
        out, ws = _check_attention(pr, b, pos, q, counts, H, dtype, rp, n, split=split, scale=0.01)
    assert torch.isfinite(out.float()).all() and float(out.float().abs().max()) > 2.0 ** 115
    assert ws is not None or n < 1000
