"""GPU: attention and its gradients where there is nothing to see, and beside
large numbers that a row or a key does not see."""
import sys

import pytest
import torch

import paper_2110_04175_amd as rs
from paper_2110_04175_amd import layer

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,keys,heads,kv,width", [(1000, 0, 1, 1, 16), (700, 0, 6, 2, 200), (20000, 0, 4, 4, 64),
                                                        (0, 1000, 4, 1, 64), (0, 300, 2, 2, 256)])
def test_many_rows_without_keys(tokens, keys, heads, kv, width, dtype):
    """Rows of which each sees nothing, keys that nothing sees: zeros, and an lse of
    -infinity."""
    announce(f"attention of {tokens} rows and {keys} keys, {dtype}")
    q = torch.ones(2, tokens, heads, width, dtype=dtype, device="cuda")
    k = torch.ones(2, keys, kv, width, dtype=dtype, device="cuda")
    starts, none = (torch.tensor([0, at], dtype=torch.int32, device="cuda") for at in (tokens, keys))
    for ranges in (None, layer.attention_ranges(starts, tokens, none, keys)):
        out, lse = layer.attention(q, k, k, ranges)
        assert (out == 0).all() and (lse == -float("inf")).all()
        grads = layer.attention_backward(q, q, k, k, out, lse, ranges)
        for g, x in zip(grads, (q, k, k)):
            assert g.shape == x.shape and (g == 0).all()


def normal(gen, *shape, std=1.0, dtype=torch.float32):
    return torch.empty(*shape).normal_(0.0, std, generator=gen).cuda().to(dtype)


def everything(q, k, v, do, ranges):
    out, lse = layer.attention(q, k, v, ranges)
    return (out, lse, *layer.attention_backward(do, q, k, v, out, lse, ranges))


def packed(seed, n, t, cuts, heads, kv, width, dtype):
    """Two sequences of every worker, from cuts[0] and cuts[1] on, and padding from
    cuts[2] on."""
    gen = torch.Generator().manual_seed(seed)
    q, do = normal(gen, n, t, heads, width, dtype=dtype), normal(gen, n, t, heads, width, std=0.01, dtype=dtype)
    k, v = normal(gen, n, t, kv, width, dtype=dtype), normal(gen, n, t, kv, width, dtype=dtype)
    return q, k, v, do, layer.attention_ranges(torch.tensor(cuts, dtype=torch.int32, device="cuda"), t)


def same(got, want, rows, what):
    """Rows of out, lse, dq, dk and dv, bit for bit."""
    for name, a, b in zip(("out", "lse", "dq", "dk", "dv"), got, want):
        a, b = (x[:, :, rows] if name == "lse" else x[:, rows] for x in (a, b))
        assert torch.equal(a, b), (what, name, int((a != b).sum()), a.numel())


SIZES = [
    # n, t, cuts, heads, kv, width
    (1, 40, [0, 17, 33], 1, 1, 16),           # one tile of few rows
    (2, 300, [0, 130, 261], 4, 2, 64),        # few rows, keys in parts
    (2, 300, [0, 130, 261], 4, 2, 100),
    (1, 700, [0, 400, 690], 4, 1, 80),        # gradients of k and v in parts of rows
    (1, 1200, [0, 650, 1111], 6, 2, 200),     # the same, one after the other
    (16, 600, [0, 320, 590], 4, 2, 48),       # tiles of many rows
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_large_values_and_gradients_that_are_not_seen(size, dtype):
    """Values of 6e4 in padding, values a hundred and gradients a million times as
    large in the other sequence: the first sequence's results keep their bits."""
    announce(f"attention beside large values {size} {dtype}")
    n, t, cuts, heads, kv, width = size
    q, k, v, do, ranges = packed(3, *size, dtype)
    want = everything(q, k, v, do, ranges)
    v[:, cuts[2]:] = 6e4
    v[:, cuts[1]:cuts[2]] *= 100
    do[:, cuts[1]:] *= 1e6
    assert all(torch.isfinite(x).all() for x in (v, do))
    same(everything(q, k, v, do, ranges), want, slice(0, cuts[1]), "the first sequence")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_large_scores_that_are_not_seen(size, dtype):
    """Queries and keys fifty times as large in padding and in the other sequence:
    scores there pass the first one's by thousands, which keeps its bits."""
    announce(f"attention beside large scores {size} {dtype}")
    q, k, v, do, ranges = packed(6, *size, dtype)
    cut = size[2][1]
    want = everything(q, k, v, do, ranges)
    q[:, cut:] *= 50
    k[:, cut:] *= 50
    got = everything(q, k, v, do, ranges)
    same(got, want, slice(0, cut), "the first sequence")
    assert all(torch.isfinite(x[:, cut:size[2][2]]).all() for x in got[:1] + got[2:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_later_tokens_with_large_scores(size, dtype):
    """As above, within one sequence: tokens from the middle of a tile on, which the
    earlier ones do not see."""
    announce(f"attention before large scores {size} {dtype}")
    q, k, v, do, _ = packed(7, *size, dtype)
    late = size[1] * 2 // 3 // 32 * 32 + 20
    assert late < size[1]
    want = everything(q, k, v, do, None)
    q[:, late:] *= 50
    k[:, late:] *= 50
    same(everything(q, k, v, do, None)[:3], want[:3], slice(0, late), "the earlier tokens")


@pytest.mark.parametrize("width", [64, 128, 200])
def test_heads_of_other_keys_that_are_large(width):
    """In binary16 a key head's values and its queries' gradients take no bits from
    another's, nor one token's gradient from those of other tokens' queries."""
    announce(f"attention beside large heads width={width}")
    q, k, v, do, ranges = packed(4, 2, 200, [0, 100, 200], 4, 2, width, torch.float16)
    want = everything(q, k, v, do, ranges)
    v[:, :, 1] *= 5e3
    do[:, :, 2:] *= 1e5
    got = everything(q, k, v, do, ranges)
    for a, b in zip(got[:3], want[:3]):
        h = 1 if a.dim() == 3 else 2
        assert torch.equal(a.narrow(h, 0, 2), b.narrow(h, 0, 2))
    for a, b in zip(got[3:], want[3:]):
        assert torch.equal(a[:, :, :1], b[:, :, :1])
    # One token's gradient: the gradients of the other tokens' queries are their own.
    do[:, 37, :2] *= 1000
    assert torch.isfinite(do).all()
    again = everything(q, k, v, do, ranges)
    rows = [i for i in range(200) if i != 37]
    assert torch.equal(again[2][:, rows], got[2][:, rows])


@pytest.mark.parametrize("width", [32, 64, 128, 256])
def test_small_weights_beside_large_values(width):
    """binary16: a sequence's values and gradients are of ordinary size, the other
    worker's thousands of times as large, and padding holds 6e4.  Its gradients are
    sums of terms ds k and ds q.  u is half a step, 2^-11; a weight is off by d as
    its score, its row's sum and exponential are, dout . out by 2 u + d, and ds is
    rounded by u: (3 u + 4 d) of a term's size before it cancels; a sum over two heads'
    rows adds 800 steps of 2^-24, the result u and 2^-24 of its own.  What ds has below
    2^-14 of its held value is off by 2^-25 of 2^13 of the column's largest: 2^-38 of
    |dout| |v|, which the sizes' d exceeds."""
    announce(f"attention in binary16 beside large values width={width}")
    t, dtype, u = 500, torch.float16, 2.0 ** -11
    q, k, v, do, ranges = packed(5, 2, t, [0, 400, 470], 2, 1, width, dtype)
    v[1] *= 5e3
    do[1] *= 1e4
    v[:, 470:] = 6e4
    do[:, 470:] = 6e4
    got = everything(q, k, v, do, ranges)
    rows = slice(0, 400)
    seen = torch.ones(400, 400, dtype=torch.bool).tril()
    qs, ks, vs, ds_ = (x[0, rows].double().cpu() for x in (q, k, v, do))
    c = width ** -0.5
    dk = torch.zeros(400, width, dtype=torch.float64)
    size_k = torch.zeros_like(dk)
    for h in range(2):
        s = (qs[:, h] @ ks[:, 0].T * c).masked_fill(~seen, -torch.inf)
        p = s.softmax(1)
        dp = ds_[:, h] @ vs[:, 0].T
        flow = p * (dp - (p * dp).sum(1, keepdim=True))
        most = p * (ds_[:, h].abs() @ vs[:, 0].abs().T + (p * (ds_[:, h].abs() @ vs[:, 0].abs().T)).sum(1, keepdim=True))
        d = 2 * (width + 8) * 2.0 ** -24 * c * (qs[:, h].abs() @ ks[:, 0].abs().T).max() + (400 + 32) * 2.0 ** -24
        dq, size_q = c * flow @ ks[:, 0], c * most @ ks[:, 0].abs()
        off = (3 * u + 4 * d) * size_q + u * dq.abs() + 2.0 ** -24
        assert ((got[2][0, rows, h].double().cpu() - dq).abs() <= off).all(), h
        dk += c * flow.T @ qs[:, h]
        size_k += c * most.T @ qs[:, h].abs() * (1 + 4 * d / (3 * u) + 800 * 2.0 ** -24 / (3 * u))
    off = 3 * u * size_k + u * dk.abs() + 2.0 ** -24
    assert ((got[3][0, rows, 0].double().cpu() - dk).abs() <= off).all()


def test_heads_of_no_width_are_refused():
    """By the call, as every other width out of range."""
    announce("attention of no width")
    x = torch.zeros(1, 2, 1, 0, device="cuda")
    with pytest.raises(rs.RelaySumError, match="width"):
        layer.attention(x, x, x)
    with pytest.raises(rs.RelaySumError, match="width"):
        layer.attention_backward(x, x, x, x, x, torch.zeros(1, 1, 2, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,n", [(1, 1), (300, 64)])
def test_the_largest_values(tokens, n, dtype):
    """Values near 2^119 / keys, of few rows and of many, whose scores rise slowly
    from key to key, so that references stay behind: results are the values."""
    announce(f"attention of the largest values {tokens} {n} {dtype}")
    keys, width = 300, 16
    big = 2.0 ** 119 / keys * 0.99
    q = torch.ones(n, tokens, 1, width, dtype=dtype, device="cuda")
    k = (torch.arange(keys, device="cuda") * 2.0 ** -8).view(1, keys, 1, 1).expand(n, keys, 1, width).to(dtype).contiguous()
    v = torch.full((n, keys, 1, width), big, dtype=dtype, device="cuda")
    out, _ = layer.attention(q, k, v, causal=False, scale=1.0)
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]
    assert ((out.double() / v[0, 0, 0, 0].double() - 1).abs() <= 3 * half + 700 * 2.0 ** -24).all()
