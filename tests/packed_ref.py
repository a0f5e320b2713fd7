"""Packed attention, rotary positions and losses from their formulas in float64, with error bounds."""
import numpy as np

EPS32 = 2.0 ** -24


def begins(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)


def attention(q, k, v, begin, scale):
    """q [rows][H][hd], k, v [rows][Hkv][hd] float64: (out, a bound) of every row of a sequence, NaN elsewhere.

    The bound holds for fp32 sums, without the rounding of probabilities and outputs: a score is a sum of hd
    products, each rounded at most hd + 2 times by half a step of 2^-24, and so is its product with scale
    log2(e) (ds below, with the exponential's own error of some units of 2^-22 of its argument's neighbour); a
    probability errs by its score's and the maximum's, relative to it; a weighted sum of L values adds L + 64
    roundings, the normaliser as many."""
    rows, H, hd = q.shape
    out = np.full((rows, H, hd), np.nan)
    bound, weight = np.full((rows, H, 1), np.nan), np.full((rows, H, hd), np.nan)
    G = H // k.shape[1]
    for b, e in zip(begin[:-1], begin[1:]):
        L = e - b
        if L == 0:
            continue
        late = np.triu(np.ones((L, L), bool), 1)
        for h in range(H):
            kk, vv = k[b:e, h // G], v[b:e, h // G]
            s = q[b:e, h] @ kk.T * scale
            size = np.abs(q[b:e, h]) @ np.abs(kk).T * abs(scale)
            s[late] = -np.inf
            p = np.exp(s - s.max(axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            out[b:e, h] = p @ vv
            weight[b:e, h] = p @ np.abs(vv)
            ds = (hd + 8) * EPS32 * np.where(late, 0.0, size).max(axis=1, keepdims=True) + 2.0 ** -20
            bound[b:e, h] = 2.0 * ds + 2.0 * (L + 64) * EPS32
    return out, bound * weight, weight


def turn(x, heads, hd, rot, layout, pos, cos, sin):
    """x [rows][heads * hd] float64 with each head's first rot values turned; and the bound of one fp32 evaluation."""
    y = x.reshape(len(x), heads, hd).copy()
    c, s = cos[pos].astype(np.float64)[:, None], sin[pos].astype(np.float64)[:, None]
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == 0 else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = y[..., lo].copy(), y[..., hi].copy()
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    bound = np.zeros_like(y)
    bound[..., lo] = 2 * EPS32 * (np.abs(a * c) + np.abs(b * s))
    bound[..., hi] = 2 * EPS32 * (np.abs(b * c) + np.abs(a * s))
    return y.reshape(x.shape), bound.reshape(x.shape)


def loss(logits, tokens, begin):
    """Mean next-token cross entropy of one half, logits float64 [rows][V]."""
    total, count = 0.0, 0
    for b, e in zip(begin[:-1], begin[1:]):
        for t in range(b, e - 1):
            x = logits[t]
            total += x.max() + np.log(np.exp(x - x.max()).sum()) - x[min(max(tokens[t + 1], 0), len(x) - 1)]
            count += 1
    return total / count if count else np.nan


def beams(logits, score, hist, length, eos, kept):
    """One prompt's step: logits float64 [b][V], score [b], hist [b][>= length].  (values, beams, tokens), largest
    first, of equal ones the lowest (beam, token); NaN first."""
    V = logits.shape[1]
    val = np.empty((len(score), V))
    for j, x in enumerate(logits):
        s = float(score[j])
        with np.errstate(all="ignore"):
            m = x.max()
            lse = m + np.log(np.exp(x - m).sum())
        if np.isnan(s) or s == np.inf:
            val[j] = np.nan
        elif eos >= 0 and length > 0 and hist[j][length - 1] == eos:
            val[j] = -np.inf
            val[j, eos] = s
        else:
            val[j] = s + (x - lse) if np.isfinite(lse) else np.nan
            if s == -np.inf and np.isfinite(lse):
                val[j] = -np.inf
    flat = val.reshape(-1)
    rank = np.where(np.isnan(flat), np.inf, flat)
    at = np.argsort(-rank, kind="stable")[:kept]
    return flat[at], at // V, at % V
