"""Performance cases of batches whose sequences differ in length, and of the step of a beam search.

A program that fine-tunes on real text packs its sequences one behind the other: it rotates the queries and keys
at each row's own token index (`zoact_rope_at`), attends within each sequence (`zoact_attention_packed`) and takes
the next-token loss over the rows that have a next token in their sequence (`zoact_linear_xent_packed` with the
head's product, `zoact_xent_packed` from stored logits).  A program that answers with beams selects the next
candidates from the logits (`zoact_beam_select`).  Layer shapes are those of the decoders in synth.

`run` makes those calls where `own` is true, else it computes them with elementary torch operations.
"""
import math

import torch

own = False
DEV = "cuda"

# heads of the decoders in synth, and others of each grouping: (H, Hkv)
HEADS = [(32, 8), (32, 8), (40, 40), (4, 4), (14, 2), (16, 8)]


def listed():
    return [
        # the tiny fp32 model on eight short sequences: latency
        {"name": "attend_tiny_fp32", "kind": "attend", "H": 4, "Hkv": 4, "hd": 32, "dtype": "fp32", "n": 8, "lo": 1,
         "hi": 65},
        # the ordinary fine-tuning batch, both halves stacked: 2 x 16 sequences of very unequal length
        {"name": "attend_batch_llama", "kind": "attend", "H": 32, "Hkv": 8, "hd": 128, "dtype": "bf16", "n": 32,
         "lo": 33, "hi": 510},
        # heads without grouping, sequences up to OPT's largest position
        {"name": "attend_batch_opt", "kind": "attend", "H": 40, "Hkv": 40, "hd": 128, "dtype": "bf16", "n": 10,
         "lo": 200, "hi": 2011},
        # one long document among thirty short ones
        {"name": "attend_skewed", "kind": "attend", "H": 32, "Hkv": 8, "hd": 128, "dtype": "bf16", "n": 31, "lo": 5,
         "hi": 12001, "one_long": True},
        # an fp32 model at lengths past the small ones
        {"name": "attend_fp32", "kind": "attend", "H": 16, "Hkv": 8, "hd": 64, "dtype": "fp32", "n": 6, "lo": 100,
         "hi": 1501},
        # single tokens of 48 sequences far into their texts, q|k of one row each: latency
        {"name": "rope_tokens_48", "kind": "rope", "heads": 40, "hd": 128, "rot": 128, "layout": "half",
         "dtype": "bf16", "rows": 48, "n_pos": 131072},
        # a packed batch, the first half of each head rotated in pairs of neighbours
        {"name": "rope_part_pairs", "kind": "rope", "heads": 40, "hd": 128, "rot": 64, "layout": "interleaved",
         "dtype": "bf16", "rows": 16411, "n_pos": 4096},
        # the first step of one prompt of the tiny model, one row to four beams: latency
        {"name": "beams_first_tiny", "kind": "beams", "n": 1, "beams_in": 1, "beams": 4, "vocab": 512, "length": 0,
         "dtype": "fp32", "ended": 0.0, "masked": 0.0},
        # four beams of each of 32 prompts over the Llama vocabulary, some ended, 100 tokens so far
        {"name": "beams_32x4_llama", "kind": "beams", "n": 32, "beams_in": 4, "beams": 4, "vocab": 128256,
         "length": 100, "dtype": "fp32", "ended": 0.1, "masked": 0.0},
        # many beams of three prompts over the OPT vocabulary, a third of it masked out
        {"name": "beams_3x16_opt", "kind": "beams", "n": 3, "beams_in": 16, "beams": 16, "vocab": 50272, "length": 17,
         "dtype": "fp32", "ended": 0.2, "masked": 0.34},
        # the tiny fp32 model's loss from its logits
        {"name": "loss_tiny_fp32", "kind": "loss", "head": False, "n": 7, "lo": 1, "hi": 80, "vocab": 512, "d": 0},
        # the Llama head with its loss on two halves of 16 sequences
        {"name": "loss_head_llama", "kind": "loss", "head": True, "n": 16, "lo": 8, "hi": 180, "vocab": 128256,
         "d": 4096},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "rope", "beams", "beams", "loss"])
    if kind == "attend":
        H, Hkv = rng.choice(HEADS)
        c = {"kind": kind, "H": H, "Hkv": Hkv, "hd": rng.choice([32, 64, 128, 128]),
             "dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"]), "n": _log_int(rng, 1, 64)}
        one = c["n"] > 2 and rng.random() < 0.2
        # products of all sequences stay below those of the longest listed case (a tenth of them in fp32)
        most = 12001 ** 2 * 32 * 128 / (H * c["hd"]) / (10 if c["dtype"] == "fp32" else 1)
        hi = _log_int(rng, 1, max(2, min(12001, int(math.sqrt(most / (2 if one else c["n"]))))))
        c.update({"lo": rng.randint(0, hi), "hi": hi})
        if one:
            c["one_long"] = True
            c["lo"] = min(c["lo"], 1 + hi // c["n"])
        return c
    if kind == "rope":
        hd = rng.choice([32, 64, 128, 128])
        heads = rng.choice([1, 5, 8, 16, 40])
        return {"kind": kind, "heads": heads, "hd": hd, "rot": rng.choice([hd, hd, hd // 2, 24, 10]),
                "layout": rng.choice(["half", "interleaved"]), "dtype": rng.choice(["bf16", "bf16", "fp32"]),
                "rows": _log_int(rng, 1, 16411 * 20 // heads * 128 // hd // 2), "n_pos": _log_int(rng, 64, 131072)}
    if kind == "beams":
        beams = rng.randint(1, 16)
        first = rng.random() < 0.2
        vocab = max(_log_int(rng, 100, 128256), 4 * beams)
        n = _log_int(rng, 1, max(2, min(64, 128 * 128256 // vocab // beams)))
        return {"kind": kind, "n": n, "beams_in": 1 if first else beams, "beams": beams, "vocab": vocab,
                "length": 0 if first else _log_int(rng, 1, 500), "dtype": rng.choice(["fp32", "fp32", "bf16"]),
                "ended": 0.0 if first else rng.choice([0.0, 0.15]), "masked": rng.choice([0.0, 0.0, 0.5])}
    head = rng.random() < 0.6
    n = _log_int(rng, 1, 32)
    vocab, d = rng.choice([(128256, 4096), (50272, 5120), (50272, 1024), (1008, 256)]) if head else \
        (_log_int(rng, 16, 60000), 0)
    most = (1500 if head else min(4000, 30000000 // vocab)) // n
    hi = max(2, _log_int(rng, 2, max(3, most)))
    return {"kind": kind, "head": head, "n": n, "lo": rng.randint(0, hi), "hi": hi, "vocab": vocab, "d": d}


# ------------------------------------------------------------------ sizes
def _lens(case):
    """Lengths of the sequences: spread between lo and hi in a mixed order, or one of hi and the rest up to
    twenty times lo."""
    n, lo, hi = case["n"], case["lo"], case["hi"]
    if n == 1:
        return [hi]
    if case.get("one_long"):
        rest = [lo + (lo * 19 * i) // n for i in range(n - 1)]
        return rest[:n // 2] + [hi] + rest[n // 2:]
    vals = [lo + round((hi - lo) * (i / (n - 1)) ** 2) for i in range(n)]
    return [vals[(i * 37 + 11) % n] if math.gcd(37, n) == 1 else vals[n - 1 - i] for i in range(n)]


def _esize(case):
    return 4 if case["dtype"] == "fp32" else 2


def _type(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def work(case):
    kind = case["kind"]
    if kind == "attend":
        lens, H, hkv, hd = _lens(case), case["H"], case["Hkv"], case["hd"]
        return {"bytes": sum(lens) * (2 * H + 2 * hkv) * hd * _esize(case),
                "flops": sum(4 * H * hd * (L * (L + 1) // 2) for L in lens)}
    if kind == "rope":
        values = case["rows"] * case["heads"] * case["hd"]
        turned = case["rows"] * case["heads"] * case["rot"]
        table = min(case["rows"], case["n_pos"]) * case["rot"] * 4
        return {"bytes": 2 * values * _esize(case) + table + 4 * case["rows"], "flops": 3 * turned}
    if kind == "beams":
        rows = case["n"] * case["beams_in"]
        kept = case["n"] * case["beams"]
        return {"bytes": rows * case["vocab"] * _esize(case) + kept * (case["length"] * 8 + 16),
                "flops": 3 * rows * case["vocab"]}
    rows, V, d = sum(_lens(case)), case["vocab"], case["d"]
    if case["head"]:
        return {"bytes": V * d * 2 + 2 * rows * d * 2, "flops": 2 * 2 * rows * V * d}
    return {"bytes": 2 * rows * V * 4, "flops": 2 * rows * V * 3}


# ------------------------------------------------------------------ inputs
class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(int(seed) * 2654435761 % (1 << 62) + 7)

    def normal(self, shape, std=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=torch.float32).mul_(std).to(dtype)

    def ints(self, lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=self.g, device=DEV, dtype=torch.int32)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device=DEV)


def _begin(lens):
    b = [0]
    for L in lens:
        b.append(b[-1] + L)
    return torch.tensor(b, dtype=torch.int32, device=DEV)


def _tables(n_pos, rot, theta=5.0e5):
    """Angles of all positions, in 64 bits, as cosines and sines in 32."""
    j = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    ang = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * theta ** (-2.0 * j / rot)
    return torch.cos(ang).float(), torch.sin(ang).float()


def prepare(case, seed):
    g, kind = _Gen(seed), case["kind"]
    s = {"case": case}
    if own:
        from paper_2607_01125_amd import zoact as Z
    if kind == "attend":
        H, hkv, hd, lens = case["H"], case["Hkv"], case["hd"], _lens(case)
        rows = sum(lens)
        s["lens"], s["begin"] = lens, _begin(lens)
        # one fused q|k|v row per token, as the projection leaves it; scores of standard deviation 2
        qkv = g.normal((max(rows, 1), (H + 2 * hkv) * hd))
        qkv[:, :H * hd] *= 2.0
        qkv = qkv.to(_type(case))[:rows]
        s["q"], s["k"], s["v"] = qkv[:, :H * hd], qkv[:, H * hd:(H + hkv) * hd], qkv[:, (H + hkv) * hd:]
        s["scale"] = float(torch.tensor(1.0 / math.sqrt(hd), dtype=torch.float32))
        if own:
            s["out"] = torch.empty(rows, H * hd, dtype=_type(case), device=DEV)
            s["seqs"] = Z.Packed(s["begin"], rows, max(lens))
    elif kind == "rope":
        rows, width = case["rows"], case["heads"] * case["hd"]
        # queries and keys of the fused row, the values behind them
        s["x"] = g.normal((rows, width + 8 * case["hd"]), dtype=_type(case))[:, :width]
        s["pos"] = g.ints(0, case["n_pos"], (rows,))
        s["cos"], s["sin"] = _tables(case["n_pos"], case["rot"])
        if own:
            s["out"] = torch.empty(rows, width, dtype=_type(case), device=DEV)
            s["layout"] = Z.ROPE_HALF if case["layout"] == "half" else Z.ROPE_INTERLEAVED
    elif kind == "beams":
        n, bi, V, length = case["n"], case["beams_in"], case["vocab"], case["length"]
        logits = g.normal((n * bi, V), 2.5)
        if case["masked"]:
            logits[:, g.uniform((V,)) < case["masked"]] = -math.inf
        s["logits"] = logits.to(_type(case))
        s["eos"] = 2
        cap = length + 1 + length // 4
        s["hist"] = g.ints(3, V, (n, bi, cap))
        if length:
            s["hist"][:, :, length - 1] = torch.where(g.uniform((n, bi)) < case["ended"], 2, s["hist"][:, :, length - 1])
        # summed log probabilities of beams that compete: far down, near one another
        s["score"] = -3.0 * length - 2.0 * g.uniform((n, bi)) if length else torch.zeros(n, bi, device=DEV)
        if own:
            b = case["beams"]
            s["to"] = Z.Beams.alloc(n, b, cap, DEV)
            s["from"] = Z.Beams(s["score"], s["hist"])
            s["token"] = torch.empty(n * b, dtype=torch.int32, device=DEV)
            s["src"] = torch.empty(n * b, dtype=torch.int32, device=DEV)
            nb = Z.beam_workspace_bytes(n, bi, b, V)
            s["ws"] = torch.empty(nb, dtype=torch.uint8, device=DEV)
    else:
        lens, V = _lens(case), case["vocab"]
        rows = sum(lens)
        s["lens"], s["begin"] = lens, _begin(lens)
        s["tokens"] = g.ints(0, V, (rows,))
        if case["head"]:
            s["x"], s["w"] = g.normal((2 * rows, case["d"]), dtype=torch.bfloat16), \
                g.normal((V, case["d"]), 0.02, torch.bfloat16)
        else:
            s["logits"] = g.normal((2, rows, V), 2.0)
        if own:
            s["seqs"] = Z.Packed(s["begin"], rows, max(lens))
            s["loss"] = torch.empty(2, device=DEV)
            if case["head"]:
                s["layer"] = Z.Linear(s["w"], case["d"], V)
                s["pert"] = Z.Pert(0, 0, 0, 0.0)
                s["ws"] = torch.empty(Z.linear_xent_workspace_bytes(rows, V), dtype=torch.uint8, device=DEV)
            else:
                s["ws"] = torch.empty(Z.loss_workspace_bytes(), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    return (_OWN if own else _PLAIN)[kind](state)


def _own_attend(s):
    from paper_2607_01125_amd import zoact as Z
    c = s["case"]
    Z.attention_packed(s["seqs"], s["q"], s["k"], s["v"], s["out"], c["H"], c["Hkv"], c["hd"], s["scale"])
    return s["out"]


def _own_rope(s):
    from paper_2607_01125_amd import zoact as Z
    Z.rope_at(s["x"], s["out"], s["case"]["heads"], s["case"]["hd"], s["pos"], s["cos"], s["sin"], s["layout"])
    return s["out"]


def _own_beams(s):
    from paper_2607_01125_amd import zoact as Z
    L = s["case"]["length"]
    Z.beam_select(s["logits"], s["from"], L, s["eos"], s["to"], s["token"], s["src"], s["ws"])
    return s["to"].score, s["to"].hist[:, :, :L + 1], s["token"], s["src"]


def _own_loss(s):
    from paper_2607_01125_amd import zoact as Z
    if s["case"]["head"]:
        Z.linear_xent_packed(s["layer"], None, s["x"], s["tokens"], s["seqs"], None, s["pert"], s["loss"], s["ws"])
    else:
        Z.xent_packed(s["logits"], s["tokens"], s["seqs"], s["loss"], s["ws"])
    return s["loss"]


def _plain_attend(s):
    c = s["case"]
    H, hkv, hd, t = c["H"], c["Hkv"], c["hd"], _type(c)
    G = H // hkv
    out = torch.empty(sum(s["lens"]), H * hd, dtype=t, device=DEV)
    r0 = 0
    for L in s["lens"]:
        if L == 0:
            continue
        r1 = r0 + L
        k = s["k"][r0:r1].float().view(L, hkv, hd).permute(1, 2, 0).contiguous()
        v = s["v"][r0:r1].float().view(L, hkv, hd).transpose(0, 1).contiguous()
        q = s["q"][r0:r1].float().view(L, hkv, G, hd).permute(1, 2, 0, 3)
        step = max(1, min(L, (1 << 27) // (H * L)))
        for a in range(0, L, step):
            b = min(a + step, L)
            x = torch.matmul(q[:, :, a:b].reshape(hkv, G * (b - a), hd), k[:, :, :b]).view(hkv, G, b - a, b)
            x *= s["scale"]
            late = torch.arange(b, device=DEV)[None, :] > torch.arange(a, b, device=DEV)[:, None]
            x.masked_fill_(late, -math.inf)
            x -= x.amax(dim=-1, keepdim=True)
            x.exp_()
            total = x.sum(dim=-1, keepdim=True)
            o = torch.matmul(x.view(hkv, G * (b - a), b), v[:, :b]).view(hkv, G, b - a, hd) / total
            out[r0 + a:r0 + b] = o.permute(2, 0, 1, 3).reshape(b - a, H * hd).to(t)
        r0 = r1
    return out


def _plain_rope(s):
    c = s["case"]
    rows, heads, hd, rot = c["rows"], c["heads"], c["hd"], c["rot"]
    x = s["x"].float().view(rows, heads, hd)
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    y = x.clone()
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return y.to(_type(c)).view(rows, heads * hd)


def _plain_beams(s):
    c = s["case"]
    n, bi, b, V, L, eos = c["n"], c["beams_in"], c["beams"], c["vocab"], c["length"], s["eos"]
    # (in 64 bits: candidates of different beams are compared)
    x = s["logits"].double().view(n, bi, V)
    top = x.amax(dim=2, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(dim=2, keepdim=True))
    val = s["score"].double()[:, :, None] + (x - lse)
    if L:
        ended = s["hist"][:, :, L - 1] == eos
        stay = torch.full((V,), -math.inf, dtype=torch.float64, device=DEV)
        stay[eos] = 0.0
        val = torch.where(ended[:, :, None], s["score"].double()[:, :, None] + stay, val)
    val = val.view(n, bi * V)
    score, at = [], []
    for _ in range(b):              # the largest left, the first of equal ones
        i = val.argmax(dim=1, keepdim=True)
        at.append(i)
        score.append(val.gather(1, i))
        val.scatter_(1, i, -math.inf)
    at, score = torch.cat(at, 1), torch.cat(score, 1)
    parent, tok = at // V, (at % V).to(torch.int32)
    hist = torch.cat([s["hist"][:, :, :L].gather(1, parent[:, :, None].expand(-1, -1, L)), tok[:, :, None]], dim=2)
    src = (parent + torch.arange(n, device=DEV)[:, None] * b).to(torch.int32)
    return score.float(), hist, tok.reshape(-1), src.reshape(-1)


def _plain_loss(s):
    rows = sum(s["lens"])
    live = torch.tensor([t for t, last in _rows(s["lens"]) if not last], dtype=torch.int64, device=DEV)
    nxt = s["tokens"].long()[live + 1][:, None]
    out = []
    for h in range(2):
        if s["case"]["head"]:
            x = torch.matmul(s["x"][h * rows:(h + 1) * rows][live].float(), s["w"].float().t())
        else:
            x = s["logits"][h][live]
        top = x.amax(dim=1, keepdim=True)
        lse = top + torch.log(torch.exp(x - top).sum(dim=1, keepdim=True))
        out.append((lse - x.gather(1, nxt)).double().mean())
    return torch.stack(out).float()


def _rows(lens):
    """(row, whether it is its sequence's last) of all sequences."""
    t = 0
    for L in lens:
        for i in range(L):
            yield t, i == L - 1
            t += 1


_OWN = {"attend": _own_attend, "rope": _own_rope, "beams": _own_beams, "loss": _own_loss}
_PLAIN = {"attend": _plain_attend, "rope": _plain_rope, "beams": _plain_beams, "loss": _plain_loss}


# ------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return _EXACT[case["kind"]](case, s)


def _exact_attend(case, s):
    H, hkv, hd = case["H"], case["Hkv"], case["hd"]
    out = torch.empty(sum(s["lens"]), H * hd, dtype=torch.float64, device=DEV)
    r0 = 0
    for L in s["lens"]:
        for h in range(H):
            g = h // (H // hkv)
            q = s["q"][r0:r0 + L, h * hd:(h + 1) * hd].double()
            k = s["k"][r0:r0 + L, g * hd:(g + 1) * hd].double()
            v = s["v"][r0:r0 + L, g * hd:(g + 1) * hd].double()
            for a in range(0, L, 4096):
                b = min(a + 4096, L)
                p = q[a:b] @ k[:b].t() * s["scale"]
                p = torch.exp(p - torch.amax(p, dim=1, keepdim=True))
                p = torch.tril(p, diagonal=a)
                # (the largest score may be a later token's: what is left is far from underflow in 64 bits)
                out[r0 + a:r0 + b, h * hd:(h + 1) * hd] = (p @ v[:b]) / p.sum(dim=1, keepdim=True)
        r0 += L
    return out


def _exact_rope(case, s):
    rows, heads, hd, rot = case["rows"], case["heads"], case["hd"], case["rot"]
    x = s["x"].double().view(rows, heads, hd)
    p = s["pos"].long()
    turn = torch.complex(s["cos"][p].double(), s["sin"][p].double())[:, None, :]
    part = x[..., :rot]
    if case["layout"] == "half":
        z = torch.complex(part[..., :rot // 2].contiguous(), part[..., rot // 2:].contiguous()) * turn
        new = torch.cat([z.real, z.imag], dim=-1)
    else:
        z = torch.view_as_complex(part.reshape(rows, heads, rot // 2, 2).contiguous()) * turn
        new = torch.view_as_real(z).reshape(rows, heads, rot)
    return torch.cat([new, x[..., rot:]], dim=-1).reshape(rows, heads * hd)


def _exact_beams(case, s):
    n, bi, b, V, L, eos = case["n"], case["beams_in"], case["beams"], case["vocab"], case["length"], s["eos"]
    score = torch.empty(n, b, dtype=torch.float64, device=DEV)
    hist = torch.empty(n, b, L + 1, dtype=torch.int32, device=DEV)
    src = torch.empty(n, b, dtype=torch.int32, device=DEV)
    for i in range(n):
        cand = []                   # (minus the value, beam, token): the order that decides
        for j in range(bi):
            sc = float(s["score"][i, j])
            if L and int(s["hist"][i, j, L - 1]) == eos:
                cand.append((-sc, j, eos))
                continue
            lp = torch.log_softmax(s["logits"][i * bi + j].double(), dim=0) + sc
            order = torch.sort(lp, descending=True, stable=True)
            cand += [(-v, j, t) for v, t in zip(order.values[:b].tolist(), order.indices[:b].tolist())]
        for m, (v, j, t) in enumerate(sorted(cand)[:b]):
            score[i, m], src[i, m] = -v, i * b + j
            hist[i, m, :L] = s["hist"][i, j, :L]
            hist[i, m, L] = t
    return score, hist, hist[:, :, L].reshape(-1), src.reshape(-1)


def _exact_loss(case, s):
    rows, out = sum(s["lens"]), []
    for h in range(2):
        total, count, r0 = torch.zeros((), dtype=torch.float64, device=DEV), 0, 0
        for L in s["lens"]:
            if L > 1:
                a = h * rows + r0
                x = (s["x"][a:a + L - 1].double() @ s["w"].double().t() if case["head"] else
                     s["logits"][h, r0:r0 + L - 1].double())
                lp = x - torch.logsumexp(x, dim=1, keepdim=True)
                total -= lp.gather(1, s["tokens"][r0 + 1:r0 + L].long()[:, None]).sum()
                count += L - 1
            r0 += L
        out.append(total / count)
    return torch.stack(out)


_EXACT = {"attend": _exact_attend, "rope": _exact_rope, "beams": _exact_beams, "loss": _exact_loss}
