"""Plain 64-bit implementations of the layer operators on 8-bit rows, one
entry at a time from their definitions; numpy arrays in and out."""
from __future__ import annotations

import numpy as np

GROUP = 128
NOT_A_NUMBER = -128


def stride_of(width: int) -> int:
    return -(-width // GROUP) * GROUP


def exponent(a: float) -> int:
    """The smallest e >= -126 with a <= 127 * 2^e; -128 for what is no number."""
    if not np.isfinite(a):
        return NOT_A_NUMBER
    e = -126
    while a > 127 * 2.0 ** e:
        e += 1
    return e


def pack(v, group=0):
    """(codes, exps) of v[n][rows][width]."""
    n, rows, width = v.shape
    s = stride_of(width)
    span = group or s
    codes = np.zeros((n, rows, s), np.int8)
    exps = np.zeros((n, rows, s // span), np.int8)
    for i in range(n):
        for t in range(rows):
            for k in range(s // span):
                part = v[i, t, k * span:min((k + 1) * span, width)].astype(np.float64)
                e = exponent(np.max(np.abs(part))) if part.size else -126
                exps[i, t, k] = e
                if e != NOT_A_NUMBER:
                    codes[i, t, k * span:k * span + part.size] = np.rint(part * 2.0 ** -e)
    return codes, exps


def values(codes, exps, width):
    """What packed rows stand for."""
    span = codes.shape[2] // exps.shape[2]
    e = np.repeat(exps.astype(np.int64), span, axis=2)
    v = np.ldexp(codes.astype(np.float64), np.where(e == NOT_A_NUMBER, 0, e))
    return np.where(e == NOT_A_NUMBER, np.nan, v)[:, :, :width]


def rmsnorm(s, weight, eps):
    """(y, rstd) of the rows s[n][tokens][width]."""
    s = s.astype(np.float64)
    rstd = 1.0 / np.sqrt(np.mean(s * s, axis=2) + eps)
    return s * rstd[:, :, None] * weight.astype(np.float64)[:, None, :], rstd


def rmsnorm_backward(dy, dsum, s, rstd, weight):
    """(ds, weight gradient) at the given s and rstd."""
    dy, s = dy.astype(np.float64), s.astype(np.float64)
    xh = s * rstd.astype(np.float64)[:, :, None]
    u = dy * weight.astype(np.float64)[:, None, :]
    dot = np.mean(u * xh, axis=2, keepdims=True)
    ds = rstd.astype(np.float64)[:, :, None] * (u - xh * dot)
    if dsum is not None:
        ds = ds + dsum.astype(np.float64)
    return ds, np.sum(dy * xh, axis=1)


def linear(x, w):
    """y[n][t][c] = sum_k x[n][t][k] w[n][c][k]."""
    return np.einsum("ntk,nck->ntc", x.astype(np.float64), w.astype(np.float64))


def linear_backward(dy, x, w):
    """(dx, dw) of linear."""
    dy = dy.astype(np.float64)
    return (np.einsum("ntc,nck->ntk", dy, w.astype(np.float64)),
            np.einsum("ntc,ntk->nck", dy, x.astype(np.float64)))


def sigmoid(f):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-f))


def blocknorm(z, gate, residual, post_weight, scale, eps):
    """(sum before it is rounded, the size of what is added to residual,
    post_rstd); what follows is rmsnorm of the rounded sum."""
    z = z.astype(np.float64)
    u, post_rstd = rmsnorm(z, post_weight, eps)
    g = 1.0 if gate is None else sigmoid(gate.astype(np.float64))
    branch = scale.astype(np.float64)[:, None, None] * g * u
    return residual.astype(np.float64) + branch, np.abs(branch), post_rstd


def blocknorm_backward(dy, dsum, z, gate, s, post_rstd, rstd, post_weight, scale, weight, size=np.asarray):
    """(ds, dz, dgate, weight, post weight and scale gradients) at the given s
    and statistics.  With size=np.abs every term is taken as large as it is:
    what roundings are measured against."""
    f8 = np.float64
    dy, z, s, w, pw = (size(v.astype(f8)) for v in (dy, z, s, weight[:, None, :], post_weight[:, None, :]))
    sc = size(scale.astype(f8)[:, None, None])
    sign = -1.0 if size is np.asarray else 1.0
    inv, pinv = rstd.astype(f8)[:, :, None], post_rstd.astype(f8)[:, :, None]
    sh, zh = s * inv, z * pinv
    u = dy * w
    ds = inv * (u + sign * sh * np.mean(u * sh, axis=2, keepdims=True))
    if dsum is not None:
        ds = size(dsum.astype(f8)) + ds
    g, rest = (1.0, 0.0) if gate is None else (sigmoid(gate.astype(f8)), sigmoid(-gate.astype(f8)))
    v = ds * sc * g * pw
    dz = pinv * (v + sign * zh * np.mean(v * zh, axis=2, keepdims=True))
    dgate = None if gate is None else ds * sc * zh * pw * g * rest
    return (ds, dz, dgate, np.sum(dy * sh, axis=1), np.sum(ds * sc * g * zh, axis=1),
            np.sum(ds * g * zh * pw, axis=(1, 2)))
