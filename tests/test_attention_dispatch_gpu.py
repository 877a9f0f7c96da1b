"""GPU: attention's gradients where key tiles are ordered by what sees them, and where
a key head's rows are split over workgroups, against 64 bits.

Tolerances as those of one row after the other.  u is half a step of the type; a
weight is off by D = 2 (width + 8) 2^-24 c |q| |k| + (keys + 32) 2^-24 (its score, its
row's sum, exponentials), and by u where it enters a product; sums over rows add
rows * 2^-24.  Sizes are those of a result's terms before they cancel:
  out  (u + 2 D) size + u |out|          dv  (u + 2 D + rows 2^-24) size + u |dv|
  dq   (3 u + 4 D) size + u |dq|         dk  (3 u + 4 D + rows 2^-24) size + u |dk|
(dout . out is off by 2 u + D, ds is rounded by u.)  In binary16 what is held below
2^-14 is off by 2^-25: 2^-40 of a weight, 2^-37 of the largest |dout| |v|, a term."""
import sys

import numpy as np
import pytest
import torch

from oracle import attention as plain
from paper_2110_04175_amd import layer

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


def wide(q, k, v, do, ranges, c):
    """(out, dq, dk, dv) and the sizes of their terms in 64 bits, a head at a time;
    what is not finite is taken as 0."""
    q, k, v, do = (torch.nan_to_num(x.double(), 0.0, 0.0, 0.0) for x in (q, k, v, do))
    n, tokens, heads, width = q.shape
    keys, kv = k.shape[1:3]
    got = [torch.zeros_like(x) for x in (q, q, k, v, q, q, k, v)]
    out, dq, dk, dv, so, sq, sk, sv = got
    at = torch.arange(keys, device=q.device)
    for i in range(n):
        r = ranges[i if ranges.shape[0] > 1 else 0]
        seen = (at >= r[:, :1]) & (at < r[:, 1:])
        some = seen.any(1, keepdim=True)
        for h in range(heads):
            g = h // (heads // kv)
            qs, d, ks, vs = q[i, :, h], do[i, :, h], k[i, :, g], v[i, :, g]
            s = torch.where(seen, c * (qs @ ks.T.contiguous()), -torch.inf)
            p = torch.where(some, torch.where(some, s, 0.0).softmax(1), 0.0)
            dp, most = d @ vs.T.contiguous(), d.abs() @ vs.abs().T.contiguous()
            ds = c * p * (dp - (p * dp).sum(1, keepdim=True))
            mag = c * p * (most + (p * most).sum(1, keepdim=True))
            pt, dst, magt = p.T.contiguous(), ds.T.contiguous(), mag.T.contiguous()
            out[i, :, h], so[i, :, h] = p @ vs, p @ vs.abs()
            dq[i, :, h], sq[i, :, h] = ds @ ks, mag @ ks.abs()
            dk[i, :, g] += dst @ qs
            sk[i, :, g] += magt @ qs.abs()
            dv[i, :, g] += pt @ d
            sv[i, :, g] += pt @ d.abs()
    return got[:4], got[4:]


def check(q, k, v, do, ranges, causal=True, rows=slice(None)):
    """Results of the rows (and keys of these places) that `rows` names."""
    n, tokens, heads, width = q.shape
    keys, t, u, c = k.shape[1], q.dtype, ROUND[q.dtype], width ** -0.5
    out, lse = layer.attention(q, k, v, ranges, causal)
    got = (out, *layer.attention_backward(do, q, k, v, out, lse, ranges, causal))
    if ranges is None:
        ranges = torch.from_numpy(plain.default_ranges(1, tokens, keys, causal).copy()).cuda()
    want, size = wide(q, k, v, do, ranges, c)

    def norm(x):
        return float(torch.nan_to_num(x.double(), 0.0, 0.0, 0.0).square().sum(-1).max().sqrt())

    d = 2 * (width + 8) * ULP * c * norm(q) * norm(k) + (keys + 32) * ULP
    sums, half = tokens * (heads // k.shape[2]) * ULP, t == torch.float16
    terms = max(keys, tokens * heads // k.shape[2])
    tiny_s = (2.0 ** -37 if half else 2.0 ** -117) * terms * norm(do) * norm(v) * c * max(norm(q), norm(k))
    tiny_p = (2.0 ** -40 if half else 2.0 ** -117) * terms * max(norm(do), norm(v))
    offs = [(u + 2 * d, 2.0 ** -117 * keys * norm(v)), (3 * u + 4 * d, tiny_s), (3 * u + 4 * d + sums, tiny_s),
            (u + 2 * d + sums, tiny_p)]
    for g, w, s, (rel, tiny), what in zip(got, want, size, offs, ("out", "dq", "dk", "dv")):
        g, w, s = g[:, rows].double(), w[:, rows], s[:, rows]
        assert torch.isfinite(g).all(), what
        off = rel * s + u * w.abs() + TINY[t] + tiny
        bad = (g - w).abs() > off
        assert not bad.any(), (what, int(bad.sum()), float((g - w).abs()[bad].max()), bad.nonzero()[:3].tolist())


def normal(seed, *shape, std=1.0, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    return torch.empty(*shape).normal_(0.0, std, generator=gen).cuda().to(dtype)


def heads(seed, n, t, h, kv, width, dtype):
    return (normal(seed, n, t, h, width, dtype=dtype), normal(seed + 1, n, t, kv, width, dtype=dtype),
            normal(seed + 2, n, t, kv, width, dtype=dtype), normal(seed + 3, n, t, h, width, std=0.1, dtype=dtype))


def cuts(seed, n, t, count):
    """Starts of sequences of very different lengths, a few of none, padding behind."""
    rng = np.random.default_rng(seed)
    at = np.sort((rng.random((n, count - 1)) ** 2 * t).astype(np.int32), 1)
    ends = rng.integers(t - 40, t + 1, (n, 1), dtype=np.int32)
    at = np.concatenate([rng.integers(0, 5, (n, 1), dtype=np.int32), at.clip(5, t - 40), ends], 1)
    return torch.from_numpy(at).cuda()


def test_the_oracle():
    """In 64 bits a head at a time is the same as a row at a time."""
    q, k, v, do = (x.cpu() for x in heads(1, 2, 30, 4, 2, 8, torch.float32))
    r = layer.attention_ranges(cuts(2, 2, 30 + 40, 3).clamp(max=30), 30)
    got, size = wide(*(x.cuda() for x in (q, k, v, do)), r, 0.3)
    want = plain.attention(*(x.numpy() for x in (q, k, v)), r.cpu().numpy(), 0.3, do.numpy())
    for a, b in zip(got + size, (want[0], *want[3], want[2], *want[4])):
        assert np.abs(a.cpu().numpy() - b).max() < 1e-12


# 160 key heads of 5 tiles: more workgroups than run at once.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [16, 96, 136])
@pytest.mark.parametrize("shared", [False, True])
def test_tiles_of_keys_in_order(shared, width, dtype):
    """Ranges of every worker's own, or one set for all of them."""
    announce(f"attention gradients in order shared={shared} width={width} {dtype}")
    n, t = 40, 520
    starts = cuts(3, n, t, 6)
    check(*heads(4, n, t, 8, 4, width, dtype), layer.attention_ranges(starts[0] if shared else starts, t))


@pytest.mark.parametrize("causal", [False, True])
def test_ranges_in_any_order(causal):
    """Windows and ranges that reach outside or are empty; tiles that nothing sees."""
    announce(f"attention gradients, any ranges, in order {causal}")
    n, t = 40, 520
    rng = np.random.default_rng(5)
    lo = np.where(rng.random((n, t, 1)) < 0.5, np.arange(t)[None, :, None] - 60, rng.integers(-20, 250, (n, t, 1)))
    hi = np.where(rng.random((n, t, 1)) < 0.1, -3, lo + rng.integers(-5, 120, (n, t, 1)))
    if causal:
        hi = np.where(hi > 0, np.minimum(hi, 200), hi)
    r = torch.from_numpy(np.concatenate([lo, hi], 2).astype(np.int32)).cuda()
    check(*heads(6, n, t, 4, 4, 32, torch.bfloat16), r)


@pytest.mark.parametrize("dtype", TYPES)
def test_more_tiles_than_are_ordered(dtype):
    """300 workers of 8 tiles of keys."""
    announce(f"attention gradients of many tiles {dtype}")
    n, t = 300, 1000
    check(*heads(7, n, t, 1, 1, 16, dtype), layer.attention_ranges(cuts(8, n, t, 4), t))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [64, 100, 200, 256])
@pytest.mark.parametrize("n,t,h,kv", [(1, 700, 2, 1), (2, 333, 6, 2), (1, 2100, 1, 1)])
def test_rows_in_parts(n, t, h, kv, width, dtype):
    """Few key heads with many rows: dk and dv are sums of workgroups' parts."""
    announce(f"attention gradients in parts {n} {t} {h} {kv} width={width} {dtype}")
    args = heads(9, n, t, h, kv, width, dtype)
    check(*args, None)
    check(*args, layer.attention_ranges(cuts(10, n, t, 4), t))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [64, 100, 200])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_seen_beside_parts(bad, width, dtype):
    """What is not finite in padding and in a second sequence, with gradients of k
    and v in parts: the first sequence's are as without it."""
    announce(f"attention gradients in parts beside {bad} width={width} {dtype}")
    n, t, cut, end = 2, 700, 443, 650
    q, k, v, do = heads(11, n, t, 2, 1, width, dtype)
    ranges = layer.attention_ranges(torch.tensor([0, cut, end], dtype=torch.int32, device="cuda"), t)
    for x in (q, k, v, do):
        x[0, 600:, :, 3] = bad
        x[1, end:] = bad
    check(q, k, v, do, ranges, rows=slice(0, cut))
    out, lse = layer.attention(q, k, v, ranges)
    for x in (out, *layer.attention_backward(do, q, k, v, out, lse, ranges)):
        assert torch.isfinite(x[1]).all() and (x[1, end:] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_seen_beside_the_order(dtype):
    announce(f"attention gradients in order beside NaN {dtype}")
    n, t, cut = 40, 520, 260
    q, k, v, do = heads(12, n, t, 4, 4, 32, dtype)
    starts = torch.tensor([[0, cut, 450 + i] for i in range(n)], dtype=torch.int32, device="cuda")
    for i in (0, 7, 39):
        for x in (q, k, v, do):
            x[i, 400:] = float("nan")
    check(q, k, v, do, layer.attention_ranges(starts, t), rows=slice(0, cut))
