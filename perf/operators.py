"""Performance cases of answering with a fine-tuned decoder: what a program that generates tokens has the
library do, beside the whole-sequence forward of the fine-tuning step.

A program holds an INT4 backbone (or a tiny fp32 model), the trained coefficients, and a paged key/value
cache held in 8 bits with one scale for each block of 16 tokens and head.  Per token it multiplies a few
rows with packed weights (`zoact_linear_rows`), rotates and quantises the new keys and values into the
cache (`zoact_cache_append`) and attends over it (`zoact_attention_cache`); between tokens it reserves,
forks, frees and compacts pages (`zoact_cache_extend`, `_fork`, `_free`, `_compact`).  The same calls
with more rows take a prompt.  Layer shapes are those of the decoders in synth; batches run from one
sequence to 64, lengths from one token to 131,072.

`run` makes those calls where `own` is true, else it computes them with elementary torch operations.
"""
import math

import torch

own = False
DEV = "cuda"
PAGE, BLOCK = 64, 16

# the packed layers of the two model shapes: name -> (d_in, d_out, epilogue, bias, residual, plain range)
LAYERS = {
    "llama_qkv": (4096, 6144, "none", False, False, (0, 0)),
    "llama_o": (4096, 4096, "none", False, True, (0, 0)),
    "llama_gate_up": (4096, 28672, "swiglu", False, False, (0, 0)),
    "llama_down": (14336, 4096, "none", False, True, (0, 0)),
    "opt_qkv": (5120, 15360, "none", True, False, (5120, 10240)),
    "opt_out": (5120, 5120, "none", True, True, (0, 0)),
    "opt_fc1": (5120, 20480, "relu", True, False, (0, 0)),
    "opt_fc2": (20480, 5120, "none", True, True, (0, 0)),
}


def listed():
    return [
        # one token of one sequence through an o projection with its residual: latency
        {"name": "rows_o_1", "kind": "rows", "layer": "llama_o", "rows": 1, "r": 32, "f32_out": False},
        # one token through gate|up with SwiGLU, the largest layer
        {"name": "rows_gate_up_1", "kind": "rows", "layer": "llama_gate_up", "rows": 1, "r": 32, "f32_out": False},
        # a ragged batch of 13 sequences through OPT's fc2 (bias, residual, rank 64)
        {"name": "rows_fc2_13", "kind": "rows", "layer": "opt_fc2", "rows": 13, "r": 64, "f32_out": False},
        # 48 sequences through the fused q|k|v
        {"name": "rows_qkv_48", "kind": "rows", "layer": "llama_qkv", "rows": 48, "r": 32, "f32_out": False},
        # the new token's keys and values of 32 sequences in the middle of their blocks, rotary
        {"name": "append_32x1", "kind": "append", "H": 32, "Hkv": 8, "hd": 128, "dtype": "bf16", "n": 32, "lo": 300,
         "hi": 2000, "new": 1, "rope": True},
        # four prompts of about 2000 tokens into an empty cache, OPT's 40 heads
        {"name": "append_prompts_opt", "kind": "append", "H": 40, "Hkv": 40, "hd": 128, "dtype": "bf16", "n": 4,
         "lo": 0, "hi": 0, "new": 2011, "rope": False},
        # the tiny fp32 model, eight short sequences: latency
        {"name": "attend_tiny_fp32", "kind": "attend", "H": 4, "Hkv": 4, "hd": 32, "dtype": "fp32", "n": 8, "lo": 1,
         "hi": 65, "new": 1, "rope": True},
        # the ordinary batch: one token of 48 sequences of very unequal length
        {"name": "attend_48_ragged", "kind": "attend", "H": 32, "Hkv": 8, "hd": 128, "dtype": "bf16", "n": 48, "lo": 70,
         "hi": 8000, "new": 1, "rope": True},
        # one token of one long sequence: the length is all there is to split
        {"name": "attend_1x131071", "kind": "attend", "H": 32, "Hkv": 8, "hd": 128, "dtype": "bf16", "n": 1,
         "lo": 131070, "hi": 131070, "new": 1, "rope": True},
        # parts of three prompts behind what the cache holds already, OPT's heads (no grouping)
        {"name": "attend_chunk_opt", "kind": "attend", "H": 40, "Hkv": 40, "hd": 128, "dtype": "bf16", "n": 3,
         "lo": 500, "hi": 1500, "new": 333, "rope": False},
        # the first step of a beam search, two layers' pages: four beams of each of eight prompts, one token reserved,
        # so that every beam copies its prompt's last page
        {"name": "pages_beams_32", "kind": "beams", "prompts": 8, "beams": 4, "len": 1000, "layers": 2, "Hkv": 8,
         "hd": 128},
        # half of 64 sequences ended: their pages go back and the rest moves together
        {"name": "pages_compact_64", "kind": "compact", "n": 64, "lo": 100, "hi": 3000, "layers": 2, "Hkv": 8,
         "hd": 128},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rows", "rows", "append", "attend", "attend", "beams", "compact"])
    if kind == "rows":
        layer = rng.choice(sorted(LAYERS))
        return {"kind": kind, "layer": layer, "rows": _log_int(rng, 1, 64), "r": rng.choice([0, 5, 16, 32, 64]),
                "f32_out": rng.random() < 0.3}
    hkv, group = rng.choice([(8, 4), (8, 4), (40, 1), (4, 2), (2, 7)])
    heads = {"H": hkv * group, "Hkv": hkv, "hd": rng.choice([32, 64, 128, 128]),
             "dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"]), "rope": rng.random() < 0.6}
    if kind in ("append", "attend"):
        n = _log_int(rng, 1, 64)
        new = 1 if rng.random() < 0.6 else _log_int(rng, 2, 300)
        # tokens times heads of all sequences stay below those of the longest listed case, and so do
        # the products of a chunk of new rows
        cap = 131072 * 8 // hkv // n
        if new > 1:
            cap = min(cap, 3 * 1800 * 333 * 40 // (hkv * group * new * n))
        hi = _log_int(rng, 1, max(cap, 2))
        return {"kind": kind, "n": n, "new": new, "lo": rng.randint(0, hi), "hi": hi, **heads}
    heads = {"Hkv": hkv, "hd": heads["hd"], "layers": rng.randint(1, 3)}
    if kind == "beams":
        return {"kind": kind, "prompts": rng.randint(1, 8), "beams": rng.randint(2, 5), "len": _log_int(rng, 1, 1000),
                **heads}
    hi = _log_int(rng, 64, 3000)
    return {"kind": kind, "n": rng.randint(2, 64), "lo": rng.randint(1, hi), "hi": hi, **heads}


# ------------------------------------------------------------------ sizes
def _lens(case):
    """Tokens each sequence holds before the call, spread between lo and hi, in a mixed order."""
    n, lo, hi = case["n"], case["lo"], case["hi"]
    if n == 1:
        return [hi]
    vals = [lo + round((hi - lo) * (i / (n - 1)) ** 2) for i in range(n)]
    return [vals[(i * 37 + 11) % n] if math.gcd(37, n) == 1 else vals[n - 1 - i] for i in range(n)]


def _news(case):
    """New rows of each sequence: `new`, or a ragged share of it from the second sequence on."""
    new = case["new"]
    return [max(1, new - (i * new) // (3 * case["n"])) for i in range(case["n"])]


def _pages(tokens):
    return -(-tokens // PAGE)


def _esize(case):
    return 4 if case.get("dtype") == "fp32" else 2


def work(case):
    kind = case["kind"]
    if kind == "rows":
        d_in, d_out, epi, bias, res, plain = LAYERS[case["layer"]]
        rows, r, out = case["rows"], case["r"], d_out // 2 if epi == "swiglu" else d_out
        adapted = d_out - (plain[1] - plain[0])
        b = d_out * d_in // 2 + d_out * (d_in // 128) * 2 + rows * (d_in + r) * 2 + adapted * r * 2
        b += (d_out * 2 if bias else 0) + (rows * d_out * 2 if res else 0) + rows * out * (4 if case["f32_out"] else 2)
        return {"bytes": b, "flops": 2 * rows * (d_out * d_in + adapted * r)}
    if kind == "append":
        rows, cols = sum(_news(case)), case["Hkv"] * case["hd"]
        held = sum((L % BLOCK) for L in _lens(case))
        b = 2 * cols * (rows * _esize(case) + rows + 2 * held)
        return {"bytes": b, "flops": rows * cols * (10 if case["rope"] else 6)}
    if kind == "attend":
        b = f = 0
        for L, c in zip(_lens(case), _news(case)):
            n = L + c
            b += 2 * case["Hkv"] * (n * case["hd"] + 4 * -(-n // BLOCK))
            b += 2 * c * case["H"] * case["hd"] * _esize(case)
            f += 4 * case["H"] * case["hd"] * (c * L + c * (c + 1) // 2)
        return {"bytes": b, "flops": f}
    page = 2 * case["layers"] * case["Hkv"] * (PAGE * case["hd"] + 16)
    if kind == "beams":
        n, L = case["prompts"] * case["beams"], case["len"]
        copied = n if L % PAGE else 0          # the prompt keeps its own last page
        return {"bytes": 2 * copied * page + 4 * n * 4 * _pages(L), "flops": n * _pages(L)}
    lens = _lens(case)
    kept = sum(_pages(L) for L in lens[1::2])
    first = _layout_pages(lens)
    moved = sum(1 for i, L in enumerate(lens) if i % 2 for p in first[i] if p >= kept)
    return {"bytes": 2 * moved * page + 8 * sum(map(_pages, lens)), "flops": 4 * sum(map(_pages, lens))}


def _layout_pages(lens):
    """Page numbers of each sequence, handed out in turn as growing sequences take them."""
    pages, nxt = [[] for _ in lens], 0
    for j in range(max(map(_pages, lens))):
        for i, L in enumerate(lens):
            if j < _pages(L):
                pages[i].append(nxt)
                nxt += 1
    return pages


# ------------------------------------------------------------------ seeded inputs
class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed) * 104729 + 5)

    def normal(self, shape, std=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=torch.float32).mul_(std).to(dtype)

    def int8(self, shape):
        """Quantised normal values: the largest of a block near 127."""
        out = torch.empty(shape, dtype=torch.int8, device=DEV)
        flat = out.view(-1)
        for i in range(0, flat.numel(), 1 << 28):
            part = flat[i:i + (1 << 28)]
            part.copy_(torch.randn(part.numel(), generator=self.g, device=DEV).mul_(36.0).clamp_(-127, 127).round_())
        return out

    def bytes(self, shape):
        return torch.randint(0, 256, shape, generator=self.g, device=DEV, dtype=torch.uint8)


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _rope_tables(n_pos, hd, theta=5.0e5):
    inv = theta ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)
    ang = torch.arange(n_pos, dtype=torch.float64)[:, None] * inv[None, :]
    return torch.cos(ang).float().to(DEV), torch.sin(ang).float().to(DEV)


def _pools(g, layers, n_pages, hkv, hd, empty=False):
    s = {"k": g.int8((layers, n_pages, hkv, PAGE, hd)) if not empty else
         torch.zeros((layers, n_pages, hkv, PAGE, hd), dtype=torch.int8, device=DEV),
         "v": g.int8((layers, n_pages, hkv, hd, PAGE)) if not empty else
         torch.zeros((layers, n_pages, hkv, hd, PAGE), dtype=torch.int8, device=DEV)}
    shp = (layers, n_pages, hkv, PAGE // BLOCK)
    s["k_scale"] = torch.exp(g.normal(shp, 0.3)).mul_(0.03)
    s["v_scale"] = torch.exp(g.normal(shp, 0.3)).mul_(0.02)
    return s


def _tables(s, pages, lens, max_pages, n_pages, slots):
    """Table, lengths and reference counts in one buffer, so that a pass puts them back with one copy."""
    host = torch.zeros(slots * max_pages + slots + n_pages, dtype=torch.int32)
    tab, ln, refs = host[:slots * max_pages].view(slots, max_pages), host[slots * max_pages:][:slots], \
        host[slots * max_pages + slots:]
    for i, (p, L) in enumerate(zip(pages, lens)):
        tab[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
        ln[i] = L
        for q in p:
            refs[q] += 1
    s["meta0"] = host.to(DEV)
    s["meta"] = s["meta0"].clone()
    m = s["meta"]
    s["table"], s["len"] = m[:slots * max_pages].view(slots, max_pages), m[slots * max_pages:][:slots]
    s["refs"] = m[slots * max_pages + slots:]


def prepare(case, seed):
    g, kind = _Gen(seed), case["kind"]
    s = {"case": case}
    if kind == "rows":
        d_in, d_out, epi, bias, res, plain = LAYERS[case["layer"]]
        rows, r = case["rows"], case["r"]
        # nibbles -7..7 in two's complement; scales as a weight of standard deviation 0.02 has them
        q = torch.randint(-7, 8, (d_out, d_in), generator=g.g, device=DEV, dtype=torch.int8).to(torch.int16) & 15
        s["w"] = (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8)
        del q
        s["sc"] = torch.exp(g.normal((d_out, d_in // 128), 0.15)).mul_(0.007).to(torch.bfloat16)
        s["x"] = g.normal((rows, d_in), dtype=torch.bfloat16)
        adapted = d_out - (plain[1] - plain[0])
        if r:
            s["p"], s["c"] = g.normal((rows, r), dtype=torch.bfloat16), g.normal((adapted * r,), 0.05, torch.bfloat16)
        s["b"] = g.normal((d_out,), 0.1, torch.bfloat16) if bias else None
        s["res"] = g.normal((rows, d_out), dtype=torch.bfloat16) if res else None
        if own:
            from paper_2607_01125_amd import zoact as Z
            s["layer"] = Z.Linear(s["w"], d_in, d_out, r, None, 0, s["b"], s["sc"], plain=plain)
            s["layer"].ws = torch.empty(Z.linear_workspace_bytes(), dtype=torch.uint8, device=DEV)
            f = torch.zeros(1, device=DEV)
            s["arena"] = Z.Arena(s["c"], f, f) if r else None
            s["y"] = torch.empty(rows, d_out // 2 if epi == "swiglu" else d_out, device=DEV,
                                 dtype=torch.float32 if case["f32_out"] else torch.bfloat16)
            s["flags"] = {"none": 0, "swiglu": Z.EPI_SWIGLU, "relu": Z.EPI_RELU}[epi]
        return s
    hkv, hd = case["Hkv"], case["hd"]
    if kind in ("append", "attend"):
        lens, news = _lens(case), _news(case)
        n, total = case["n"], sum(news)
        act = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
        counts = [_pages(L + c) for L, c in zip(lens, news)]
        n_pages = sum(counts) + 3
        perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        if kind == "append":
            perm = list(range(n_pages))      # in order: what a pass wrote is then one view of the pool
        pages, k0 = [], 0
        for c in counts:
            pages.append(perm[k0:k0 + c])
            k0 += c
        s.update(_pools(g, 1, n_pages, hkv, hd, empty=kind == "append" and case["hi"] == 0))
        _tables(s, pages, [L + c for L, c in zip(lens, news)], max(counts) + 1, n_pages, n)
        begins = [0]
        for c in news:
            begins.append(begins[-1] + c)
        s["begin"], s["pos"] = _i32(begins), _i32(lens)
        s["rope"] = _rope_tables(max(L + c for L, c in zip(lens, news)), hd) if case["rope"] else None
        s["scale"] = 1.0 / math.sqrt(hd)
        # one fused q|k|v row per token, as the projection leaves it
        width = (case["H"] + 2 * hkv) * hd
        qkv = g.normal((total, width), dtype=act)
        s["q"], s["kn"] = qkv[:, :case["H"] * hd], qkv[:, case["H"] * hd:(case["H"] + hkv) * hd]
        s["vn"] = qkv[:, (case["H"] + hkv) * hd:]
        if own:
            from paper_2607_01125_amd import zoact as Z
            s["cache"] = Z.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["len"], s["refs"])
            s["batch"] = Z.CacheBatch(s["pos"], max(news), total, row_begin=s["begin"])
            if kind == "attend":
                s["out"] = torch.empty(total, case["H"] * hd, dtype=act, device=DEV)
                s["max_len"] = max(L + c for L, c in zip(lens, news))
                nb = Z.attention_cache_workspace_bytes(s["cache"], s["batch"], case["H"], s["max_len"])
                s["ws"] = torch.empty(max(nb, 16), dtype=torch.uint8, device=DEV)
        return s
    layers = case["layers"]
    if kind == "beams":
        P, B, L = case["prompts"], case["beams"], case["len"]
        lens = [L] * P + [0] * (P * B)
        pages = _layout_pages([L] * P) + [[] for _ in range(P * B)]
        n_pages = P * _pages(L) + 2 * P * B + 5
        s.update(_pools(g, layers, n_pages, hkv, hd))
        _tables(s, pages, lens, _pages(L) + 2, n_pages, P + P * B)
        s["src"] = _i32([i // B for i in range(P * B)])
        s["dst"] = _i32([P + i for i in range(P * B)])
        s["pos"] = torch.zeros(P * B, dtype=torch.int32, device=DEV)
    else:
        lens = _lens(case)
        pages = _layout_pages(lens)
        n_pages = sum(map(len, pages)) + 7
        s.update(_pools(g, layers, n_pages, hkv, hd))
        _tables(s, pages, lens, max(map(len, pages)), n_pages, len(lens))
        s["ended"] = _i32(list(range(0, len(lens), 2)))
    s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if own:
        from paper_2607_01125_amd import zoact as Z
        s["cache"] = Z.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["len"], s["refs"])
        s["ws"] = torch.empty(Z.cache_workspace_bytes(s["cache"]), dtype=torch.uint8, device=DEV)
        s["used"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        if kind == "beams":
            s["batch"] = Z.CacheBatch(s["pos"], 1, s["dst"].numel(), slots=s["dst"], status=s["status"])
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _written(s):
    """The values that the blocks an append touched stand for: one view of each pool times its scales."""
    case, k, v = s["case"], s["k"][0], s["v"][0]
    n_pages, hkv, hd = k.shape[0], k.shape[1], k.shape[3]
    kv = k.view(n_pages, hkv, PAGE // BLOCK, BLOCK, hd) * s["k_scale"][0][..., None, None]
    # V's token 16 n + 4 g + i of a page lies at position 16 g + 4 n + i
    vv = v.view(n_pages, hkv, hd, 4, 4, 4) * s["v_scale"][0][:, :, None, None, :, None]
    return kv, vv


def _run_own(s):
    from paper_2607_01125_amd import zoact as Z
    case, kind = s["case"], s["case"]["kind"]
    if kind == "rows":
        Z.linear_rows(s["layer"], s["arena"], s["x"], s.get("p"), s["y"], residual=s["res"], flags=s["flags"])
        return s["y"]
    if kind == "append":
        Z.cache_append(s["cache"], 0, s["kn"], s["vn"], s["batch"], rope=s["rope"])
        return _written(s) + (s["k_scale"], s["v_scale"])
    if kind == "attend":
        Z.attention_cache(s["cache"], 0, s["q"], s["out"], s["batch"], case["H"], s["scale"], s["max_len"],
                          rope=s["rope"], ws=s["ws"])
        return s["out"]
    s["meta"].copy_(s["meta0"])          # every pass starts from the same tables
    if kind == "beams":
        Z.cache_fork(s["cache"], s["src"], s["dst"], s["ws"], s["status"])
        Z.cache_extend(s["cache"], s["batch"], s["ws"])
        return s["table"], s["len"], s["refs"], s["pos"], s["k"], s["v"], s["k_scale"], s["v_scale"]
    Z.cache_free(s["cache"], s["ended"], s["status"])
    Z.cache_compact(s["cache"], s["ws"], s["used"])
    return s["table"], s["len"], s["refs"], s["used"], s["k"], s["v"], s["k_scale"], s["v_scale"]


def _weights(s, dtype):
    """Values -7..7 of the packed weights, [d_out][groups][128]."""
    w = s["w"]
    lo, hi = (w & 15).to(dtype), (w >> 4).to(dtype)
    q = torch.stack([lo, hi], dim=-1).view(w.shape[0], -1, 128)
    return torch.where(q > 7, q - 16, q)


def _rotate(x, pos, rope):
    """Rotate-half of rows [rows][heads][hd] at positions pos."""
    c, sn = rope[0][pos][:, None, :].to(x.dtype), rope[1][pos][:, None, :].to(x.dtype)
    half = x.shape[-1] // 2
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * c - hi * sn, hi * c + lo * sn], dim=-1)


def _v_order():
    t = torch.arange(PAGE, device=DEV)
    return ((t >> 2) & 3) * 16 + (t >> 4) * 4 + (t & 3)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "rows":
        return _plain_rows(s)
    if kind == "append":
        _plain_append(s)
        return _written(s) + (s["k_scale"], s["v_scale"])
    if kind == "attend":
        return _plain_attend(s)
    s["meta"].copy_(s["meta0"])
    if kind == "beams":
        _plain_fork(s, s["src"].long(), s["dst"].long())
        _plain_extend(s, s["dst"].long())
        return s["table"], s["len"], s["refs"], s["pos"], s["k"], s["v"], s["k_scale"], s["v_scale"]
    _plain_free(s, s["ended"].long())
    used = _plain_compact(s)
    return s["table"], s["len"], s["refs"], used, s["k"], s["v"], s["k_scale"], s["v_scale"]


def _plain_rows(s):
    case = s["case"]
    d_in, d_out, epi, _, _, plain = LAYERS[case["layer"]]
    w = (_weights(s, torch.float32) * s["sc"].float()[:, :, None]).view(d_out, d_in)
    y = s["x"].float() @ w.t()
    if case["r"]:
        corr = s["p"].float() @ s["c"].float().view(-1, case["r"]).t()
        y[:, :plain[0]] += corr[:, :plain[0]]
        y[:, plain[1]:] += corr[:, plain[0]:]
    if s["b"] is not None:
        y += s["b"].float()
    if s["res"] is not None:
        y += s["res"].float()
    if epi == "relu":
        y = torch.relu(y)
    elif epi == "swiglu":
        gu = y.view(y.shape[0], -1, 2, 16)
        gate = gu[:, :, 0]
        y = (gate / (1 + torch.exp(-gate)) * gu[:, :, 1]).reshape(y.shape[0], -1)
    return y if case["f32_out"] else y.to(torch.bfloat16)


def _plain_append(s):
    """Every touched block of 16 tokens at once: gathered, requantised with the new rows, put back."""
    case = s["case"]
    hkv, hd = case["Hkv"], case["hd"]
    page, blk, rows, held = [], [], [], []
    base = 0
    k0 = 0
    for L, c in zip(_lens(case), _news(case)):
        for b in range(L // BLOCK, -(-(L + c) // BLOCK)):
            page.append(k0 + b * BLOCK // PAGE)
            blk.append(b % (PAGE // BLOCK))
            t = range(b * BLOCK, (b + 1) * BLOCK)
            rows.append([base + x - L if L <= x < L + c else -1 for x in t])
            held.append([x < L for x in t])
        k0 += _pages(L + c)
        base += c
    page, blk = torch.tensor(page, device=DEV), torch.tensor(blk, device=DEV)
    rows, held = torch.tensor(rows, device=DEV), torch.tensor(held, device=DEV)
    new = rows >= 0
    kn, vn = (s[n].view(-1, hkv, hd).float() for n in ("kn", "vn"))
    if s["rope"] is not None:
        pos = torch.cat([torch.arange(L, L + c, device=DEV) for L, c in zip(_lens(case), _news(case))])
        kn = _rotate(kn, pos, s["rope"])
    for x, pool, sc, is_v in ((kn, s["k"][0], s["k_scale"][0], False), (vn, s["v"][0], s["v_scale"][0], True)):
        fresh = x[rows.clamp(min=0)] * new[:, :, None, None]                  # [items][16][hkv][hd]
        s_new = fresh.abs().amax(dim=(1, 3)) / 127.0                          # [items][hkv]
        had = held.any(dim=1)
        s_old = torch.where(had[:, None], sc[page, :, blk], torch.zeros_like(s_new))
        s_new = torch.maximum(s_new, s_old)
        div = torch.where(s_new > 0, s_new, torch.ones_like(s_new))
        q = torch.round(fresh / div[:, None, :, None])
        if is_v:
            view = pool.view(-1, hkv, hd, 4, 4, 4)                            # [page][head][dim][g][block][i]
            old = view[page, :, :, :, blk].reshape(len(page), hkv, hd, 16).permute(0, 3, 1, 2)
        else:
            view = pool.view(-1, hkv, 4, BLOCK, hd)
            old = view[page, :, blk].permute(0, 2, 1, 3)
        kept = torch.round(old.float() * (s_old / div)[:, None, :, None])
        q = torch.where(new[:, :, None, None], q, torch.where(held[:, :, None, None], kept, old.float())).to(torch.int8)
        if is_v:
            view[page, :, :, :, blk] = q.permute(0, 2, 3, 1).reshape(len(page), hkv, hd, 4, 4)
        else:
            view[page, :, blk] = q.permute(0, 2, 1, 3)
        sc[page, :, blk] = s_new


def _plain_attend(s):
    case = s["case"]
    H, hkv, hd = case["H"], case["Hkv"], case["hd"]
    G, order, outs, r0 = H // hkv, _v_order(), [], 0
    for i, (L, c) in enumerate(zip(_lens(case), _news(case))):
        n = L + c
        ids = s["table"][i, :_pages(n)].long()
        k = s["k"][0][ids].permute(1, 0, 2, 3).reshape(hkv, -1, hd)[:, :n].float()
        v = s["v"][0][ids].index_select(3, order).permute(1, 0, 3, 2).reshape(hkv, -1, hd)[:, :n].float()
        ks, vs = (s[m][0][ids].permute(1, 0, 2).reshape(hkv, -1).repeat_interleave(BLOCK, 1)[:, :n]
                  for m in ("k_scale", "v_scale"))
        q = s["q"][r0:r0 + c].reshape(c, H, hd).float()
        if s["rope"] is not None:
            q = _rotate(q, torch.arange(L, n, device=DEV), s["rope"])
        q = q.view(c, hkv, G, hd).permute(1, 0, 2, 3).reshape(hkv, c * G, hd)
        sc = torch.matmul(q, k.transpose(1, 2).contiguous()) * (ks * s["scale"])[:, None, :]
        if c > 1:
            row = torch.arange(L, n, device=DEV).repeat_interleave(G)
            sc = sc.masked_fill(torch.arange(n, device=DEV)[None, :] > row[:, None], -math.inf)
        p = torch.exp(sc - sc.amax(dim=2, keepdim=True))
        o = torch.matmul(p * vs[:, None, :], v) / p.sum(dim=2, keepdim=True)
        outs.append(o.view(hkv, c, G, hd).permute(1, 0, 2, 3).reshape(c, H * hd))
        r0 += c
    return torch.cat(outs).to(s["q"].dtype)


def _named(s, slots):
    """Which table entries of the slots name a page."""
    mp = s["table"].shape[1]
    return torch.arange(mp, device=DEV)[None, :] < ((s["len"][slots] + PAGE - 1) // PAGE)[:, None]


def _count(s, slots, by):
    pages, named = s["table"][slots].long(), _named(s, slots)
    s["refs"].index_add_(0, torch.where(named, pages, torch.zeros_like(pages)).view(-1),
                         (named.to(torch.int32) * by).view(-1))


def _plain_free(s, slots):
    _count(s, slots, -1)
    s["len"][slots] = 0


def _plain_fork(s, src, dst):
    _count(s, src, 1)
    _count(s, dst, -1)
    rows, named, lens = s["table"][src], _named(s, src), s["len"][src]
    s["table"][dst] = torch.where(named, rows, s["table"][dst])
    s["len"][dst] = lens


def _plain_extend(s, slots):
    """One token more for each slot (all distinct); a shared last page is copied, but for its last holder."""
    n = slots.numel()
    L = s["len"][slots].long()
    last = s["table"][slots, (L - 1).clamp(min=0) // PAGE].long()
    part = L % PAGE != 0
    same = (last[:, None] == last[None, :]) & part[:, None] & part[None, :]
    rank = torch.tril(same, -1).sum(dim=1)
    cow = part & (rank < s["refs"][last] - 1)
    need = (cow | ~part).long()
    free = torch.nonzero(s["refs"] == 0).view(-1)
    page = free[(torch.cumsum(need, 0) - need).clamp(max=free.numel() - 1)]
    s["refs"].index_add_(0, last, -cow.to(torch.int32))
    page = page[need.bool()]
    s["refs"][page] = 1
    s["table"][slots[need.bool()], (L // PAGE)[need.bool()]] = page.to(torch.int32)
    dst = torch.full((n,), -1, device=DEV)
    dst[need.bool()] = page
    for pool in ("k", "v", "k_scale", "v_scale"):
        s[pool][:, dst[cow]] = s[pool][:, last[cow]]
    s["pos"].copy_(L)
    s["len"][slots] = (L + 1).to(torch.int32)


def _plain_compact(s):
    used = s["refs"] > 0
    n_used = used.sum()
    idx = torch.arange(used.numel(), device=DEV)
    src, dst = torch.nonzero(used & (idx >= n_used)).view(-1), torch.nonzero(~used & (idx < n_used)).view(-1)
    for pool in ("k", "v", "k_scale", "v_scale"):
        s[pool][:, dst] = s[pool][:, src]
    to = idx.clone()
    to[src] = dst
    slots = torch.arange(s["len"].numel(), device=DEV)
    s["table"].copy_(torch.where(_named(s, slots), to[s["table"].long()].to(torch.int32), s["table"]))
    s["refs"][dst] = s["refs"][src]
    s["refs"][src] = 0
    return n_used.to(torch.int32).view(1)


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    if case["kind"] == "rows":
        return _exact_rows(case, prepare(case, seed))
    if case["kind"] == "attend":
        return _exact_attend(case, prepare(case, seed))
    return None            # codes, scales and page numbers: equal in every form, or wrong


def _exact_rows(case, s):
    d_in, d_out, epi, _, _, (p0, p1) = LAYERS[case["layer"]]
    x = s["x"].double()
    y = torch.zeros(case["rows"], d_out, dtype=torch.float64, device=DEV)
    for g in range(d_in // 128):          # one group of 128 inputs at a time
        by = s["w"][:, 64 * g:64 * g + 64].to(torch.int16)
        nib = torch.empty(d_out, 128, dtype=torch.int16, device=DEV)
        nib[:, ::2], nib[:, 1::2] = by % 16, by // 16
        nib -= 16 * (nib >= 8).to(torch.int16)
        y += (x[:, 128 * g:128 * g + 128] @ nib.double().T) * s["sc"][:, g].double()
    if case["r"]:
        c = s["c"].double().view(-1, case["r"])
        rows = torch.cat([torch.arange(p0, device=DEV), torch.arange(p1, d_out, device=DEV)])
        y[:, rows] += s["p"].double() @ c.T
    for extra in (s["b"], s["res"]):
        if extra is not None:
            y += extra.double()
    if epi == "relu":
        y = y.clamp(min=0)
    if epi == "swiglu":
        f = torch.arange(d_out // 2, device=DEV)
        at = f // 16 * 32 + f % 16
        y = y[:, at] * torch.sigmoid(y[:, at]) * y[:, at + 16]
    return y


def _exact_attend(case, s):
    H, hkv, hd = case["H"], case["Hkv"], case["hd"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    r0 = 0
    for i, (L, c) in enumerate(zip(_lens(case), _news(case))):
        n = L + c
        t = torch.arange(n, device=DEV)
        page, tok = s["table"][i].long()[t // PAGE], t % PAGE
        at = tok // 4 % 4 * 16 + tok // 16 * 4 + tok % 4
        ahead = t[None, :] > torch.arange(L, n, device=DEV)[:, None]
        for h in range(H):
            j = h // (H // hkv)
            k = s["k"][0, page, j, tok].double() * s["k_scale"][0, page, j, tok // BLOCK].double()[:, None]
            v = s["v"][0, page, j, :, at].double() * s["v_scale"][0, page, j, tok // BLOCK].double()[:, None]
            q = s["q"][r0:r0 + c, h * hd:(h + 1) * hd].double()
            if s["rope"] is not None:
                co, si = s["rope"][0][L:n].double(), s["rope"][1][L:n].double()
                a, b = q[:, :hd // 2], q[:, hd // 2:]
                q = torch.cat((a * co - b * si, b * co + a * si), 1)
            z = torch.softmax((q @ k.T * s["scale"]).masked_fill(ahead, -math.inf), dim=1)
            out[r0:r0 + c, h * hd:(h + 1) * hd] = z @ v
        r0 += c
    return out
