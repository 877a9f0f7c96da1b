"""Plain 64-bit attention and its gradients from their definitions, one row
at a time; numpy arrays in and out."""
from __future__ import annotations

import numpy as np


def ranges_of(starts, tokens, key_starts, keys, causal):
    """[n][tokens][2] of packed sequences, from lists of starts of each worker."""
    out = np.zeros((len(starts), tokens, 2), np.int64)
    for i, (rows, cols) in enumerate(zip(starts, key_starts)):
        for s in range(len(rows) - 1):
            for t in range(rows[s], rows[s + 1]):
                lo, hi = cols[s], cols[s + 1]
                if causal:
                    hi -= rows[s + 1] - 1 - t
                out[i, t] = lo, max(lo, hi)
    return out


def default_ranges(n, tokens, keys, causal):
    t = np.arange(tokens)
    hi = np.clip(t + 1 + keys - tokens, 0, keys) if causal else np.full(tokens, keys)
    return np.broadcast_to(np.stack([np.zeros_like(hi), hi], 1), (n, tokens, 2))


def attention(q, k, v, ranges, scale, dout=None):
    """(out, lse), and with dout also (dq, dk, dv) and for each of the four
    results the sum of the sizes of its terms: what roundings are measured
    against."""
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    n, tokens, heads, width = q.shape
    keys, kv = k.shape[1], k.shape[2]
    out, lse = np.zeros_like(q), np.full((n, heads, tokens), -np.inf)
    size = np.zeros_like(q)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    sq, sk, sv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for i in range(n):
        for t in range(tokens):
            lo, hi = max(0, int(ranges[i, t, 0])), min(keys, int(ranges[i, t, 1]))
            if lo >= hi:
                continue
            for h in range(heads):
                g = h // (heads // kv)
                kk, vv = k[i, lo:hi, g], v[i, lo:hi, g]
                with np.errstate(all="ignore"):
                    s = scale * (kk @ q[i, t, h])
                    m = np.max(s)
                    e = np.exp(s - m)
                    p = e / np.sum(e)
                    lse[i, h, t] = m + np.log(np.sum(e))
                    out[i, t, h] = p @ vv
                    size[i, t, h] = p @ np.abs(vv)
                    if dout is None:
                        continue
                    do = dout[i, t, h].astype(np.float64)
                    dp = vv @ do
                    ds = p * (dp - p @ dp)
                    # What ds is made of, before it cancels.
                    mag = p * (np.abs(vv) @ np.abs(do) + p @ (np.abs(vv) @ np.abs(do)))
                    dq[i, t, h] = scale * (ds @ kk)
                    sq[i, t, h] = scale * (mag @ np.abs(kk))
                    dk[i, lo:hi, g] += scale * np.outer(ds, q[i, t, h])
                    sk[i, lo:hi, g] += scale * np.outer(mag, np.abs(q[i, t, h]))
                    dv[i, lo:hi, g] += np.outer(p, do)
                    sv[i, lo:hi, g] += np.outer(p, np.abs(do))
    if dout is None:
        return out, lse, size
    return out, lse, size, (dq, dk, dv), (sq, sk, sv)
