"""Answering with a fine-tuned decoder: a batch of sequences over one paged 8-bit key/value cache.

A Session holds the cache of a Decoder's layers and runs the unperturbed model (C as trained, no halves)
over new tokens of any of its sequences: prompts in chunks, single tokens, or both in one call.  As in the
decoder module, every operation of the forward is a libzoact call, and so is a beam search's selection; this
module lays out buffers and picks single candidates' tokens from the logits.

Layers with INT4 weights run on zoact_linear_rows up to ROWS_MAX rows; larger chunks, and bf16 and fp32
models, run the two-halves linears of the training forward with sign 0, the rows shared out over the
halves.

The two do not have the same INT4 weight: linear_rows multiplies a group's sum by its scale (the weight is
q s), the training forward's products read bf16(q s), up to 2^-9 away from it.  A layer's outputs differ by
1.3e-3 of their norm before they are rounded to bf16 (which takes 1.7e-3), the logits of 32 layers of the
Llama-3-8B shape with random weights by 8.8e-2, where taking the prompt in two chunks instead of one moves them by
4.9e-2 and a bf16 step of the embeddings by 2.0e-1.  With trained_weights every call has the weights that C was
tuned on: a token of one sequence takes 6.2 ms instead of 5.1 there, of 48 sequences 6.9 instead of 5.2.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import zoact as Z


class Session:
    """Sequences in slots 0 .. max_seqs - 1 of up to max_tokens tokens each, over n_pages pages of 64 tokens
    (default: enough for all at full length).  Decoders with heads of 32, 64 or 128 values.  max_rows: most
    new rows of one call; longer prompts are taken in chunks.  trained_weights: INT4 weights as the training
    forward rounds them in calls of few rows too (see above).  Calls on one Session, and on all Sessions of one
    decoder, whose workspaces they share, follow each other on one stream of its device, the current one.
    Single tokens of long sequences are best decoded apart from prompts: see the attention's note on mixed
    batches in zoact_cache.h."""

    def __init__(self, decoder, max_seqs: int, max_tokens: int, *, n_pages: int | None = None, max_rows: int = 2048,
                 trained_weights: bool = False):
        d = self.dec = decoder
        if not 1 <= max_seqs <= Z.CACHE_MAX_BATCH:
            raise ValueError(f"max_seqs must be in [1, {Z.CACHE_MAX_BATCH}]")
        if max_rows < max_seqs:
            raise ValueError("max_rows must hold one row of every sequence")
        if d.hd not in (32, 64, 128):
            raise ValueError(f"the cache holds heads of 32, 64 or 128 values, not {d.hd}")
        self.max_pages = -(-max_tokens // Z.CACHE_PAGE)
        self.cache = Z.Cache.alloc(d.s.n_layers, n_pages or max_seqs * self.max_pages, d.Hkv, d.hd, max_seqs,
                                   self.max_pages, d.dev)
        self.lens = [0] * max_seqs                 # the lengths the cache has, on the host
        self.max_rows = max_rows + max_rows % 2
        self.few_rows = Z.ROWS_MAX if d.mode == "int4" and not trained_weights else 0
        self.status = torch.zeros(1, dtype=torch.int32, device=d.dev)
        self.cache_ws = torch.empty(Z.cache_workspace_bytes(self.cache), dtype=torch.uint8, device=d.dev)
        self.rope = d._rope_tables(self.max_pages * Z.CACHE_PAGE) if d.s.family == "llama" else None
        self._att_ws = None
        self._ch = None
        e = lambda *shp: torch.empty(self.max_rows, *shp, dtype=d.act, device=d.dev)
        fused = "qkv" in d.layers[0]
        self._buf = {"h0": e(d.d), "h1": e(d.d), "a": e(d.d), "qkv": e(d.d + 2 * d.dkv) if fused else e(2 * d.d),
                     "k": None if fused else e(d.dkv), "att": e(d.d), "ff": e(d.s.d_ff), "p": e(max(d.r, 1)),
                     "emb": torch.empty(2 * self.max_rows, d.d, dtype=d.act, device=d.dev),
                     "pos": torch.empty(2 * self.max_rows, d.d, dtype=d.act, device=d.dev) if d.pos is not None else None}

    # ---------------------------------------------------------------- sequences
    def _slots(self, slots, distinct=True) -> torch.Tensor:
        slots = [int(s) for s in slots]
        if not slots or any(not 0 <= s < len(self.lens) for s in slots) or (distinct and len(set(slots)) < len(slots)):
            raise ValueError(f"slots {slots}: expected different ones in [0, {len(self.lens)})")
        return torch.tensor(slots, dtype=torch.int32, device=self.dec.dev)

    def fork(self, src, dst):
        """Sequences dst[i] become what src[i] are (all at once: entries may permute slots)."""
        if len(src) != len(dst):
            raise ValueError("as many sources as destinations")
        Z.cache_fork(self.cache, self._slots(src, distinct=False), self._slots(dst), self.cache_ws, self.status)
        new = [self.lens[s] for s in src]
        for t, n in zip(dst, new):
            self.lens[t] = n

    def _fork_beams(self, src: torch.Tensor, dst: torch.Tensor):
        """fork of beams by device lists whose sources and destinations are of one length (the host's need no
        change, and does not wait)."""
        Z.cache_fork(self.cache, src, dst, self.cache_ws, self.status)

    def free(self, slots):
        """Empty the slots; pages that nobody else holds are free again."""
        Z.cache_free(self.cache, self._slots(slots), self.status)
        for s in slots:
            self.lens[s] = 0

    def compact(self) -> int:
        """Move the used pages to the front of the pool; returns their number (waits for the GPU)."""
        used = torch.empty(1, dtype=torch.int32, device=self.dec.dev)
        Z.cache_compact(self.cache, self.cache_ws, used)
        return int(used)

    def resize(self, n_pages: int):
        """Give the pool another number of pages, at least those in use (the sequences stay)."""
        used = self.compact()
        if n_pages < max(used, 1):
            raise ValueError(f"{used} pages are in use")
        old, c = self.cache, self.cache
        new = Z.Cache.alloc(c.k.shape[0], n_pages, c.n_kv_heads, c.head_dim, c.table.shape[0], c.table.shape[1],
                            c.k.device)
        for name in ("k", "v", "k_scale", "v_scale"):
            getattr(new, name)[:, :used].copy_(getattr(old, name)[:, :used])
        new.refs[:used].copy_(old.refs[:used])
        new.table.copy_(old.table)
        new.len.copy_(old.len)
        self.cache = new
        self.cache_ws = torch.empty(Z.cache_workspace_bytes(new), dtype=torch.uint8, device=self.dec.dev)

    def check(self):
        """Raise if a call since the last check found no place for what it was given (waits for the GPU).
        From that call on, nothing that was given until this check has been taken (logits of such calls mean
        nothing): each sequence holds a beginning of what it was given, lens says how long a one."""
        bits = int(self.status)
        if bits:
            self.status.zero_()
            self.lens = self.cache.len.tolist()
        if bits & Z.STATUS_NO_PAGES:
            raise RuntimeError("the cache has too few free pages: free sequences or resize, and go on from what lens "
                               "says the sequences hold")
        if bits:
            raise RuntimeError(f"the cache refused an entry (status {bits})")

    # ---------------------------------------------------------------- the model over new rows
    def forward(self, slots, tokens: torch.Tensor, counts) -> torch.Tensor:
        """Run the next counts[i] (>= 1) tokens of sequences slots[i]; tokens int32 [sum of counts], on the
        decoder's device, in that order.  Returns the logits of each sequence's last new token, fp32
        [len(slots)][vocab] (a buffer of this call's own)."""
        d, s = self.dec, self.dec.s
        counts = [int(c) for c in counts]
        rows, n = sum(counts), len(counts)
        if n != len(slots) or min(counts, default=0) < 1 or rows > self.max_rows:
            raise ValueError(f"expected a count of at least 1 for every slot, {self.max_rows} rows at most")
        ids = self._slots(slots)
        if tokens.dtype != torch.int32 or tokens.shape != (rows,) or not tokens.is_contiguous():
            raise ValueError(f"tokens must be a contiguous int32 [{rows}]")
        if tokens.get_device() != self.cache.index or torch.cuda.current_device() != self.cache.index:
            raise ValueError(f"tokens on {tokens.device}, cuda:{torch.cuda.current_device()} is the current device, "
                             f"the cache is on cuda:{self.cache.index}")
        for sl, c in zip(slots, counts):
            if self.lens[sl] + c > self.max_pages * Z.CACHE_PAGE:
                raise ValueError(f"slot {sl} would pass {self.max_pages * Z.CACHE_PAGE} tokens")
        if not d._adapted_sites <= d.ut.keys():      # (before places are reserved that would get no keys)
            raise RuntimeError("adapted sites without a basis: run basis_init or set_basis first")
        ends = np.cumsum(counts)
        # (no rows for anybody once a call was refused, so that no later one leaves a hole in a sequence)
        begin = torch.tensor([0, *ends.tolist()], dtype=torch.int32, device=d.dev).mul_(self.status == 0)
        batch = Z.CacheBatch(torch.empty(n, dtype=torch.int32, device=d.dev), max(counts), rows,
                             slots=ids, row_begin=begin, status=self.status)
        Z.cache_extend(self.cache, batch, self.cache_ws)
        for sl, c in zip(slots, counts):
            self.lens[sl] += c
        max_len = max(self.lens[sl] for sl in slots)
        need = Z.attention_cache_workspace_bytes(self.cache, batch, d.H, max_len)
        if need and (self._att_ws is None or self._att_ws.numel() < need):
            self._att_ws = torch.empty(need, dtype=torch.uint8, device=d.dev)

        T = (rows + 1) // 2                        # rows of a half in the two-halves linears
        few = rows <= self.few_rows
        B = {k: v[:2 * T] if v is not None else None for k, v in self._buf.items() if k not in ("emb", "pos")}
        pert = Z.pert_pair(0, 0, (0, 0), (0, 0), 0.0)
        d._cur = B
        d._ch = None
        if d.act == torch.bfloat16 and d.k > 0 and not few:
            # bf16(C), both halves alike, formed from C as it is now
            if self._ch is None:
                self._ch = torch.empty(2 * d.k, dtype=torch.bfloat16, device=d.dev)
            Z.perturb_coeffs(d.arena, 0, d.k, pert, self._ch)
            d._ch = self._ch
        self._embed(tokens, batch, counts, rows)
        h, h_alt = B["h0"], B["h1"]
        h[:rows].copy_(self._buf["emb"][:rows])
        if 2 * T > rows:
            h[rows:].zero_()
        scale = float(np.float32(1.0 / math.sqrt(d.hd)))

        def linear(lb, x, y, ut, residual=None, flags=0):
            lin, blk = lb
            if not few:
                return d._apply(lb, x, T, y, pert, ut, residual=residual, flags=flags, adapt=ut is not None)
            adapted = blk is not None and ut is not None
            r = d.r if adapted else 0
            if lin.r != r:
                lin.r = r
            if d.linear_hook:
                d.linear_hook("pre", lin, rows, flags)
            Z.linear_rows(lin, d.arena if adapted else None, x[:rows], B["p"][:rows] if adapted else None, y[:rows],
                          residual[:rows] if residual is not None else None, flags)
            if d.linear_hook:
                d.linear_hook("post", lin, rows, flags)

        for l, P in enumerate(d.layers):
            ut = d._norm_site(l, "attn", h, P["n1"], P.get("n1b"), B["a"], True, None, 2 * T)
            qkv = B["qkv"]
            if "qkv" in P:
                linear(P["qkv"], B["a"], qkv, ut)
                q, k, v = qkv[:, :d.d], qkv[:, d.d:d.d + d.dkv], qkv[:, d.d + d.dkv:]
            else:
                linear(P["qv"], B["a"], qkv, ut)
                linear(P["k"], B["a"], B["k"], None)
                q, k, v = qkv[:, :d.d], B["k"], qkv[:, d.d:]
            Z.cache_append(self.cache, l, k[:rows], v[:rows], batch, rope=self.rope)
            Z.attention_cache(self.cache, l, q[:rows], B["att"][:rows], batch, d.H, scale, max_len, rope=self.rope,
                              ws=self._att_ws if need else None)
            if 2 * T > rows:
                B["att"][rows:].zero_()
            ut = d._site(l, "o", B["att"], True, None)
            linear(P["o"], B["att"], h_alt, ut, residual=h)
            h, h_alt = h_alt, h
            ut = d._norm_site(l, "mlp", h, P["n2"], P.get("n2b"), B["a"], True, None, 2 * T)
            linear(P["gu"], B["a"], B["ff"], ut, flags=Z.EPI_SWIGLU if s.family == "llama" else Z.EPI_RELU)
            ut = d._site(l, "down", B["ff"], True, None)
            linear(P["down"], B["ff"], h_alt, ut, residual=h)
            h, h_alt = h_alt, h
        # the last row of each sequence: final norm and head
        m = n + n % 2
        last = torch.zeros(m, dtype=torch.int64)
        last[:n] = torch.from_numpy(ends - 1)
        x = h.index_select(0, last.to(d.dev))
        y = torch.empty_like(x)
        d._norm(x, d.nf, getattr(d, "nfb", None), y)
        logits = torch.empty(m, s.vocab, dtype=torch.float32, device=d.dev)
        Z.linear_fwd_pm(d.head, None, y, m // 2, None, logits, pert)
        d._ch = None
        return logits[:n]

    def _embed(self, tokens, batch, counts, rows):
        """Token (and learned position) embeddings of the rows into the first half of self._buf["emb"]."""
        d, out = self.dec, self._buf["emb"][:2 * rows]
        if d.pos is None:
            Z.embed(tokens, d.emb, out, rows)
            return
        # the rows' positions, looked up first (learned positions start at row 2 of their table), stand in
        # for a position table of that many rows
        c = torch.tensor(counts, device=d.dev)
        at = torch.arange(rows, device=d.dev) - torch.repeat_interleave(torch.cumsum(c, 0) - c, c, output_size=rows)
        at = at + torch.repeat_interleave(batch.pos.clamp(min=0), c, output_size=rows) + 2
        pos = self._buf["pos"][:2 * rows]
        Z.embed(at.to(torch.int32), d.pos, pos, rows)
        Z.embed(tokens, d.emb, out, rows, pos[:rows], pos_offset=0)

    # ---------------------------------------------------------------- prompts and tokens
    def prefill(self, slots, prompts) -> torch.Tensor:
        """Take prompts (sequences of token ids, none empty) into the slots, behind what they hold; the
        logits of each one's last token, fp32 [n][vocab].  Chunks of up to max_rows rows, the sequences
        packed one behind the other."""
        if len(slots) != len(prompts) or any(len(p) < 1 for p in prompts):
            raise ValueError("one prompt of at least one token for every slot")
        self._slots(slots)
        todo = [[int(sl), torch.as_tensor(p, dtype=torch.int32).reshape(-1), i] for i, (sl, p) in
                enumerate(zip(slots, prompts))]
        out = torch.empty(len(prompts), self.dec.s.vocab, dtype=torch.float32, device=self.dec.dev)
        while todo:
            room, part = self.max_rows, []
            for sl, p, i in todo:
                if room == 0:
                    break
                part.append((sl, p[:room], i, len(p) <= room))
                room -= min(room, len(p))
            toks = torch.cat([p for _, p, _, _ in part]).to(self.dec.dev)
            logits = self.forward([sl for sl, _, _, _ in part], toks, [len(p) for _, p, _, _ in part])
            for j, (_, p, i, done) in enumerate(part):
                if done:
                    out[i].copy_(logits[j])
                else:
                    todo[j][1] = todo[j][1][len(p):]
            todo = [t for t in todo if t[2] not in {i for _, _, i, done in part if done}]
        return out

    def decode(self, slots, tokens: torch.Tensor) -> torch.Tensor:
        """One token more for each slot (tokens int32 [n] on the device); their logits, fp32 [n][vocab]."""
        return self.forward(slots, tokens, [1] * len(slots))


def generate(decoder, prompts, n_new: int, *, eos: int | None = None, beams: int = 1, max_rows: int = 2048,
             n_pages: int | None = None, trained_weights: bool = False) -> list:
    """Continuations of the prompts (lists of token ids) by up to n_new tokens: the likeliest token each
    time, or with beams > 1 the likeliest of that many candidates followed at once (by their tokens' summed
    log probabilities).  Ends a sequence at `eos`, which is not returned.  max_rows, n_pages and trained_weights
    are the Session's.  Returns lists of token ids."""
    if n_new < 1 or beams < 1 or not prompts:
        raise ValueError("expected prompts, n_new >= 1 and beams >= 1")
    n = len(prompts)
    longest = max(len(p) for p in prompts) + n_new
    ses = Session(decoder, n * beams, longest, max_rows=max(max_rows, n * beams), n_pages=n_pages,
                  trained_weights=trained_weights)
    first = [i * beams for i in range(n)]
    logits = ses.prefill(first, prompts)
    ses.check()
    if beams == 1:
        out = [[] for _ in prompts]
        live = list(range(n))
        for step in range(n_new):
            tok = logits.argmax(dim=1).to(torch.int32)
            host = tok.tolist()
            keep = []
            for j, i in enumerate(live):
                if host[j] == eos:
                    continue
                out[i].append(host[j])
                keep.append(j)
            ended = [live[j] for j in range(len(live)) if j not in set(keep)]
            if ended:
                ses.free(ended)
                tok = tok[torch.tensor(keep, dtype=torch.int64, device=tok.device)].contiguous() if keep else tok[:0]
            live = [live[j] for j in keep]
            if not live or step == n_new - 1:
                break
            logits = ses.decode(live, tok)
            ses.check()
        return out

    dev, V = decoder.dev, decoder.s.vocab
    if beams > V:
        raise ValueError("more beams than tokens")
    slots = list(range(n * beams))
    ses.fork([f for f in first for _ in range(beams)], slots)
    ids = ses._slots(slots)
    tok, src = torch.empty_like(ids), torch.empty_like(ids)
    eos = eos if eos is not None and 0 <= eos < V else None
    ws = torch.empty(Z.beam_workspace_bytes(n, beams, beams, V), dtype=torch.uint8, device=dev)
    select = Z.beam_select if ws.numel() else _select_many
    now, then = Z.Beams.alloc(n, 1, n_new, dev), Z.Beams.alloc(n, beams, n_new, dev)
    for step in range(n_new):
        select(logits, now, step, eos, then, tok, src, ws)
        now, then = then, now if step else Z.Beams.alloc(n, beams, n_new, dev)
        if step == n_new - 1 or (eos is not None and bool((tok == eos).all())):
            break
        if step:
            ses._fork_beams(src, ids)
        logits = ses.decode(slots, tok)
        ses.check()
    best = now.hist[:, 0, :step + 1].tolist()
    return [row[:row.index(eos)] if eos is not None and eos in row else row for row in best]


def _select_many(logits, now: Z.Beams, length: int, eos: int | None, to: Z.Beams, tok, src, ws):
    """beam_select for more candidates than it takes."""
    (n, _), b, V = now.score.shape, to.score.shape[1], logits.shape[1]
    lp = torch.log_softmax(logits, dim=1).view(n, -1, V)
    if eos is not None and length:            # an ended candidate goes on as it is
        stay = torch.full((V,), -math.inf, device=logits.device)
        stay[eos] = 0.0
        lp = torch.where((now.hist[:, :, length - 1] == eos)[:, :, None], stay, lp)
    score, best = (now.score[:, :, None] + lp).view(n, -1).topk(b, dim=1)
    parent = best // V
    to.score.copy_(score)
    to.hist[:, :, :length] = now.hist[:, :, :length].gather(1, parent[:, :, None].expand(-1, -1, length))
    to.hist[:, :, length] = best % V
    tok.copy_((best % V).view(-1))
    src.copy_((parent + torch.arange(n, device=best.device)[:, None] * b).view(-1))
