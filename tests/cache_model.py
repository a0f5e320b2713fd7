"""A plain model of the paged 8-bit cache: bookkeeping in Python integers, codes and scales in the float32
operations that the header states, attention in float64."""
import numpy as np

PAGE, BLOCK = 64, 16


def v_place(t):
    """Position of token t of a page in a row of V."""
    return ((t >> 2) & 3) * 16 + (t >> 4) * 4 + (t & 3)


class Model:
    def __init__(self, n_layers, n_pages, hkv, hd, n_slots, max_pages):
        self.nl, self.np, self.hkv, self.hd = n_layers, n_pages, hkv, hd
        self.k = np.zeros((n_layers, n_pages, hkv, PAGE, hd), np.int8)
        self.v = np.zeros((n_layers, n_pages, hkv, hd, PAGE), np.int8)
        self.ks = np.zeros((n_layers, n_pages, hkv, 4), np.float32)
        self.vs = np.zeros((n_layers, n_pages, hkv, 4), np.float32)
        self.table = np.zeros((n_slots, max_pages), np.int32)
        self.len = np.zeros(n_slots, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.status = 0

    # ------------------------------------------------ pages
    def held(self, slot):
        return [int(p) for p in self.table[slot, :-(-int(self.len[slot]) // PAGE)]]

    def extend(self, slots, counts):
        ok, seen = [], set()
        for s, c in zip(slots, counts):
            good = 0 <= s < len(self.len) and s not in seen and c >= 0 and \
                self.len[s] + c <= self.table.shape[1] * PAGE
            seen.add(s)
            ok.append(good)
            if not good:
                self.status |= 2
        refs, plan = self.refs.copy(), []
        for s, c, good in zip(slots, counts, ok):
            cow, grow = False, 0
            if good:
                L = int(self.len[s])
                if c and L % PAGE:
                    last = int(self.table[s, L // PAGE])
                    cow = refs[last] > 1
                    refs[last] -= cow
                grow = -(-(L + c) // PAGE) - -(-L // PAGE)
            plan.append((cow, grow))
        free = [int(p) for p in np.flatnonzero(self.refs == 0)]
        if sum(c + g for c, g in plan) > len(free):
            self.status |= 4
            return [-1] * len(slots)
        pos = []
        for s, c, good, (cow, grow) in zip(slots, counts, ok, plan):
            if not good:
                pos.append(-1)
                continue
            L = int(self.len[s])
            pos.append(L)
            if cow:
                old, new = int(self.table[s, L // PAGE]), free.pop(0)
                for a in (self.k, self.v, self.ks, self.vs):
                    a[:, new] = a[:, old]
                self.refs[old] -= 1
                self.refs[new] = 1
                self.table[s, L // PAGE] = new
            for j in range(grow):
                p = free.pop(0)
                self.refs[p] = 1
                self.table[s, -(-L // PAGE) + j] = p
            self.len[s] = L + c
        return pos

    def fork(self, src, dst):
        n = len(self.len)
        rows = [(self.held(s), int(self.len[s])) if 0 <= s < n else None for s in src]
        seen = set()
        todo = []
        for i, d in enumerate(dst):
            good = 0 <= d < n and rows[i] is not None and d not in seen
            seen.add(d)
            if not good:
                self.status |= 2
                continue
            for p in rows[i][0]:
                self.refs[p] += 1
            todo.append((i, d))
        for i, d in todo:
            for p in self.held(d):
                self.refs[p] -= 1
        for i, d in todo:
            self.table[d, :len(rows[i][0])] = rows[i][0]
            self.len[d] = rows[i][1]

    def free(self, slots):
        for s in slots:
            if not 0 <= s < len(self.len):
                self.status |= 2
                continue
            for p in self.held(s):
                self.refs[p] -= 1
            self.len[s] = 0

    def compact(self):
        used = int((self.refs > 0).sum())
        src = [p for p in range(used, self.np) if self.refs[p] > 0]
        dst = [p for p in range(used) if self.refs[p] == 0]
        for s, d in zip(src, dst):
            for a in (self.k, self.v, self.ks, self.vs):
                a[:, d] = a[:, s]
            self.refs[d], self.refs[s] = self.refs[s], 0
        to = dict(zip(src, dst))
        for slot in range(len(self.len)):
            for j, p in enumerate(self.held(slot)):
                self.table[slot, j] = to.get(p, p)
        return used

    # ------------------------------------------------ codes
    def append(self, layer, slot, pos, k, v, rope=None):
        """k, v float32 [c][hkv][hd] of one entry."""
        c = k.shape[0]
        if rope is not None:
            t = np.minimum(np.arange(pos, pos + c), rope[0].shape[0] - 1)
            co, si = rope[0][t][:, None], rope[1][t][:, None]
            h = self.hd // 2
            lo, hi = k[..., :h], k[..., h:]
            k = np.concatenate([lo * co - hi * si, hi * co + lo * si], -1)
        for b in range(pos // BLOCK, -(-(pos + c) // BLOCK)):
            p, blk = int(self.table[slot, b * BLOCK // PAGE]), b % 4
            t0, t1 = max(pos, b * BLOCK), min(pos + c, (b + 1) * BLOCK)
            for x, codes, scales, isv in ((k, self.k, self.ks, False), (v, self.v, self.vs, True)):
                new = x[t0 - pos:t1 - pos]
                for h in range(self.hkv):
                    xs = new[:, h]
                    held = b * BLOCK < pos
                    old = scales[layer, p, h, blk] if held else np.float32(0)
                    s = np.float32(np.abs(xs).max()) * np.float32(1 / 127) if np.isfinite(xs).all() else np.float32(np.nan)
                    ratio = None
                    if held:
                        if np.isnan(s) or np.isnan(old):
                            s = np.float32(np.nan)
                        elif s > old:
                            ratio = old / s
                        else:
                            s = old
                    with np.errstate(all="ignore"):
                        q = np.clip(np.rint(xs / s), -127, 127) if s > 0 else np.zeros_like(xs)
                    if ratio is not None:
                        for t in range(b * BLOCK, pos):
                            at = (layer, p, h, slice(None), v_place(t % PAGE)) if isv else (layer, p, h, t % PAGE)
                            codes[at] = np.rint(codes[at].astype(np.float32) * ratio).astype(np.int8)
                    for i, t in enumerate(range(t0, t1)):
                        at = (layer, p, h, slice(None), v_place(t % PAGE)) if isv else (layer, p, h, t % PAGE)
                        codes[at] = q[i].astype(np.int8)
                    scales[layer, p, h, blk] = s

    # ------------------------------------------------ attention
    def values(self, layer, slot, n):
        """Keys and values [n][hkv][hd] in float64 of a slot's first n tokens."""
        k, v = np.zeros((2, n, self.hkv, self.hd))
        for t in range(n):
            p, i = int(self.table[slot, t // PAGE]), t % PAGE
            k[t] = self.k[layer, p, :, i].astype(np.float64) * self.ks[layer, p, :, i // BLOCK].astype(np.float64)[:, None]
            v[t] = (self.v[layer, p, :, :, v_place(i)].astype(np.float64)
                    * self.vs[layer, p, :, i // BLOCK].astype(np.float64)[:, None])
        return k, v


def attend(q, k, v, pos, scale, rope=None):
    """q [c][H][hd] float64 over k, v [n][hkv][hd]; returns the result, the mean of |v| under the same
    weights, and the largest sum of |q k| of a visible score (for error bounds)."""
    c, H, hd = q.shape
    n, hkv = k.shape[:2]
    q = q.copy()
    if rope is not None:
        t = np.minimum(np.arange(pos, pos + c), rope[0].shape[0] - 1)
        co, si = rope[0][t].astype(np.float64)[:, None], rope[1][t].astype(np.float64)[:, None]
        lo, hi = q[..., :hd // 2].copy(), q[..., hd // 2:].copy()
        q = np.concatenate([lo * co - hi * si, hi * co + lo * si], -1)
    out, mean, mag = np.zeros((c, H, hd)), np.zeros((c, H, hd)), np.zeros((c, H, 1))
    for j in range(c):
        m = pos + j + 1
        for h in range(H):
            kk, vv = k[:m, h * hkv // H], v[:m, h * hkv // H]
            s = kk @ q[j, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[j, h], mean[j, h] = p @ vv, p @ np.abs(vv)
            mag[j, h] = (np.abs(kk) @ np.abs(q[j, h]) * scale).max()
    return out, mean, mag


def attend_bound(out, mean, mag, n, hd, fp32):
    """Largest error of the kernel's result by its own roundings.

    A score's error is that of q's f16 terms (half a step: 2^-12 relative in one term, 2^-23 in two, as the
    second rounds what is left, at most 2^-12 of q, to 2^-12 again or -- far below the column's largest --
    to a fixed 2^-39 of that), of the rotation (two roundings, 2^-23), of the fp32 sum of hd products and of
    two scale products (hd + 4 steps of at most 2^-23), all relative to sum |q k| scale = mag; the
    exponential adds 2^-21 and, for its argument's rounding in the log2 domain, 2^-23 times the score again.
    A relative error e of the weights moves the result by at most 2 e times the weighted mean of |v|.
    Weights enter the second product in the same number of terms; its sum and the normaliser's have n + 8
    steps and the joins of waves and splits 140.
    """
    term = 2.0 ** -23 if fp32 else 2.0 ** -12
    e = mag * (term + (hd + 8) * 2.0 ** -23) + 2.0 ** -21
    t = 2 * e * mean + mean * (2 * term + 2 * (n + 150) * 2.0 ** -23)
    return t + np.abs(out) * (2.0 ** -24 if fp32 else 2.0 ** -8) + 1e-30
