"""GPU: the norms around a block and their gradients against the plain 64-bit
implementation (oracle/layer.py).

Tolerances.  A row's statistics take at most min(width, 42) additions, whose
terms are not negative, and a few steps more: R = (min(width, 42) + 8) * 2^-24.
The branch that is added to residual has that, some 12 steps of its products and
its gate's exponential, and |gate| * 2^-23 from the exponent's rounding in 16-bit
types; the sum is rounded once to its type.  What follows is the norm of the
rounded sum, so it is held to the sum that came out: statistics and codes as
the plain norm's.  In the gradients every value is off by at most
(2 * min(width, 42) + 40 + 2 |gate|) * 2^-24 of the size of its terms (the oracle
again, with all of them taken positive), sums over tokens by tokens * 2^-24 more
(half of it for a sum in two levels would do), and by one rounding to their type."""
import sys

import numpy as np
import pytest
import torch

from oracle import layer as plain
from paper_2110_04175_amd import layer

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 1e-6


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def normal(seed, *shape, std=1.0, mean=0.0, dtype=torch.float32):
    g = np.random.default_rng(seed).standard_normal(shape) * std + mean
    return torch.from_numpy(g.astype(np.float32)).cuda().to(dtype)


def inputs(seed, n, t, w, dtype, gated=True):
    return dict(z=normal(seed, n, t, w, std=2.0, dtype=dtype), gate=normal(seed + 1, n, t, w, dtype=dtype) if gated else None,
                residual=normal(seed + 2, n, t, w, dtype=dtype), post_weight=normal(seed + 3, n, w, std=0.1, mean=1.0),
                scale=normal(seed + 4, n, std=0.2, mean=0.5), weight=normal(seed + 5, n, w, std=0.1, mean=1.0))


def check_forward(x, keep=True, eps=EPS):
    s, y, post_rstd, rstd, saved = got = layer.blocknorm(**x, eps=eps, keep=keep)
    n, t, w = x["z"].shape
    dtype = x["z"].dtype
    h = {k: host(v) for k, v in x.items()}
    want, branch, want_post = plain.blocknorm(h["z"], h["gate"], h["residual"], h["post_weight"], h["scale"], eps)
    rel = (min(w, 42) + 8) * ULP
    most = 0 if h["gate"] is None or dtype == torch.float32 else np.abs(h["gate"]).max(initial=0)
    np.testing.assert_allclose(host(post_rstd), want_post, rtol=rel)
    sh = host(s)
    assert (np.abs(sh - want) <= (rel + (12 + 2 * most) * ULP) * branch + ROUND[dtype] * np.abs(want) * (1 + 2 ** -7)
            + ROUND[dtype] * rel * branch + TINY[dtype]).all()
    wy, want_rstd = plain.rmsnorm(sh, h["weight"], eps)
    np.testing.assert_allclose(host(rstd), want_rstd, rtol=rel)
    if keep:
        codes, exps = plain.pack(sh, 128)
        assert np.array_equal(saved.codes.cpu().numpy(), codes) and np.array_equal(saved.exps.cpu().numpy(), exps)
    else:
        assert saved is None
    e = y.exps.cpu().numpy().astype(np.int64)
    top, slack = np.max(np.abs(wy), axis=2, keepdims=True), 1 + 2 * rel + 4 * ULP
    assert (top <= 127 * 2.0 ** e * slack).all() and ((top * slack > 127 * 2.0 ** (e - 1)) | (e == -126)).all()
    off = np.abs(plain.values(y.codes.cpu().numpy(), y.exps.cpu().numpy(), w) - wy)
    assert (off <= 0.5 * 2.0 ** e + (rel + 4 * ULP) * np.abs(wy)).all()
    assert (y.codes[:, :, w:] == 0).all()
    return got


def gradients(x, got, dy, dsum, dp=None, dsc=None, dw=None):
    n, t, w = x["z"].shape
    dp, dw = (torch.full((n, w), 9.0, device="cuda") if v is None else v for v in (dp, dw))
    dsc = torch.full((n,), 9.0, device="cuda") if dsc is None else dsc
    dz, dgate, ds = layer.blocknorm_backward(dy, dsum, x["z"], x["gate"], got[4], got[2], got[3], x["post_weight"],
                                             x["scale"], x["weight"], dp, dsc, dw)
    return ds, dz, dgate, dw, dp, dsc


def check_backward(x, got, dy, dsum):
    out = gradients(x, got, dy, dsum)
    n, t, w = x["z"].shape
    dtype = x["z"].dtype
    s = plain.values(got[4].codes.cpu().numpy(), got[4].exps.cpu().numpy(), w)
    h = {k: host(v) for k, v in x.items()}
    args = (host(dy), host(dsum), h["z"], h["gate"], s, host(got[2]), host(got[3]), h["post_weight"], h["scale"], h["weight"])
    want, size = plain.blocknorm_backward(*args), plain.blocknorm_backward(*args, size=np.abs)
    most = 0 if h["gate"] is None or dtype == torch.float32 else np.abs(h["gate"]).max(initial=0)
    rel = (2 * min(w, 42) + 40 + 2 * most) * ULP
    for i, (g, a, b) in enumerate(zip(out, want, size)):
        if a is None:
            assert g is None
            continue
        g = host(g)
        u = ROUND[dtype] if i < 3 else ULP
        sums = 0 if i < 3 else (t * (w if i == 5 else 1)) * ULP
        off = (rel + sums) * b + u * np.abs(a) + (TINY[dtype] if i < 3 else 2.0 ** -126)
        assert np.isfinite(g).all() and (np.abs(g - a) <= off).all(), (i, np.abs(g - a).max())
    return out


WIDTHS = [1, 7, 128, 129, 511, 520, 1001, 1024, 1030, 2048, 2056, 4100, 8192, 8200, 16390, 32768]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_widths(width, dtype):
    announce(f"blocknorm width={width} {dtype}")
    n, t = (3, 5) if width < 8000 else (2, 2)
    for gated in (True, False):
        x = inputs(width, n, t, width, dtype, gated)
        got = check_forward(x)
        check_backward(x, got, normal(7, n, t, width, std=0.1, dtype=dtype), normal(8, n, t, width, std=0.1, dtype=dtype))
        check_forward(x, keep=False)


@pytest.mark.parametrize("n,tokens", [(1, 1), (16, 1), (1, 1000), (7, 33), (300, 2), (3, 17)])
def test_shapes(n, tokens):
    announce(f"blocknorm n={n} tokens={tokens}")
    x = inputs(1, n, tokens, 96, torch.bfloat16)
    got = check_forward(x)
    check_backward(x, got, normal(7, n, tokens, 96, dtype=torch.bfloat16), None)


def test_no_tokens():
    announce("blocknorm of nothing")
    x = inputs(2, 2, 0, 40, torch.float16)
    got = layer.blocknorm(**x)
    assert got[0].shape == (2, 0, 40) and got[1].codes.shape == (2, 0, 128)
    out = gradients(x, got, x["z"], None)
    assert out[0].shape == (2, 0, 40) and all((g == 0).all() for g in out[3:])


@pytest.mark.parametrize("dtype", TYPES)
def test_strides(dtype):
    """Parameters and their gradients inside models of odd length, activations
    as parts of wider rows, workers inside tokens, broadcast rows."""
    announce(f"blocknorm strides {dtype}")
    n, t, w = 3, 20, 77
    x = inputs(3, n, t, w, dtype)
    dy, dsum = normal(7, n, t, w, dtype=dtype), normal(8, n, t, w, dtype=dtype)
    got = check_forward(x)
    want = check_backward(x, got, dy, dsum)
    both = torch.full((n, 4 * w + 10), 7.0, device="cuda")      # models, then gradients
    model, grads = both[:, :2 * w + 5], both[:, 2 * w + 5:]
    views = dict(post_weight=model[:, 1:1 + w], scale=model[:, 1 + w], weight=model[:, 2 + w:2 + 2 * w])
    wide = torch.zeros(n, t, 3 * w + 2, dtype=dtype, device="cuda")
    views |= dict(z=wide[:, :, 1:1 + w], gate=wide[:, :, 1 + w:1 + 2 * w], residual=wide[:, :, 2 + 2 * w:])
    for k, v in views.items():
        v.copy_(x[k])
    again = layer.blocknorm(**views)
    for a, b in zip(got[:1] + got[2:4], again[:1] + again[2:4]):
        assert torch.equal(a, b)
    assert torch.equal(got[1].codes, again[1].codes) and torch.equal(got[4].codes, again[4].codes)
    out = gradients(views, again, dy.transpose(0, 1).contiguous().transpose(0, 1), dsum,
                    grads[:, 3:3 + w], grads[:, 3 + w], grads[:, 4 + w:4 + 2 * w])
    assert all(torch.equal(a, b) for a, b in zip(want, out))
    assert (grads[:, :3] == 7).all() and (grads[:, 4 + 2 * w:] == 7).all() and torch.equal(model[:, 1 + w], x["scale"])
    one = {k: (v[:1, :1].expand(n, t, w) if v.dim() == 3 else v) for k, v in x.items()}
    check_backward(one, check_forward(one), dy, dsum)


def test_rows_that_are_special():
    """Rows of zeros, of a NaN or an infinity, far outside binary32's squares,
    and gates at both ends."""
    announce("blocknorm special rows")
    x = inputs(4, 1, 7, 256, torch.float32)
    x["z"][0, 1] = 0
    x["z"][0, 2, 9] = float("nan")
    x["z"][0, 3] *= 1e25
    x["z"][0, 4] *= 1e-30
    x["gate"][0, 5, :100] = float("inf")
    x["gate"][0, 5, 100:] = -float("inf")
    x["residual"][0, 6, 4] = float("inf")
    s, y, post_rstd, rstd, saved = layer.blocknorm(**x)
    v = layer.unpack(y, torch.float32)
    assert torch.equal(s[0, 1], x["residual"][0, 1])
    assert torch.isnan(s[0, 2]).all() and torch.isnan(v[0, 2]).all() and torch.isnan(v[0, 6]).all()
    assert torch.isfinite(s[0, [0, 1, 3, 4, 5]]).all() and torch.isfinite(v[0, [0, 1, 3, 4, 5]]).all()
    assert ((s[0, 5, 100:] - x["residual"][0, 5, 100:]).abs() < 1e-30).all()
    ok = [0, 1, 3, 5]
    z, w = host(x["z"])[:, ok], host(x["post_weight"])
    want = plain.blocknorm(z, host(x["gate"])[:, ok], host(x["residual"])[:, ok], w, host(x["scale"]), EPS)[0]
    assert np.abs(host(s)[:, ok] - want).max() < 1e-5
    dy = normal(9, 1, 7, 256)
    out = gradients(x, (s, y, post_rstd, rstd, saved), dy, None)
    fine = [0, 1, 3, 4, 5]
    for g in out[:3]:
        assert torch.isfinite(g[0, fine]).all()


def test_far_rows():
    announce("blocknorm far rows")
    n, t, w = 1, 70, 40
    far = torch.empty(n, t, 1 << 26, dtype=torch.bfloat16, device="cuda")
    x = inputs(5, n, t, w, torch.bfloat16)
    got = layer.blocknorm(**x)
    far[:, :, -w:] = x["z"]
    far[:, :, 5:5 + w] = x["gate"]
    y = x | dict(z=far[:, :, -w:], gate=far[:, :, 5:5 + w])
    again = layer.blocknorm(**y)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1].codes, again[1].codes)
    dy = normal(6, n, t, w, dtype=torch.bfloat16)
    assert all(torch.equal(a, b) for a, b in zip(gradients(x, got, dy, None), gradients(y, again, dy, None)))


def test_graphs_and_streams():
    """Two captured graphs of the whole pass, replayed in turn with new inputs
    and eager calls between, and the pass on another stream."""
    announce("blocknorm in graphs")

    def step(x, dy):
        got = layer.blocknorm(**x)
        return [got[0], got[1].codes, got[4].codes, *gradients(x, got, dy, dy)]

    made = []
    for seed, n, t, w in ((10, 4, 100, 300), (20, 2, 37, 1500)):
        x, dy = inputs(seed, n, t, w, torch.bfloat16), normal(seed + 9, n, t, w, dtype=torch.bfloat16)
        step(x, dy)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = step(x, dy)
        made.append((x, dy, g, outs))
    side = torch.cuda.Stream()
    for turn in range(3):
        for x, dy, g, outs in made:
            for i, v in enumerate([*x.values(), dy]):
                v.copy_(normal(50 * turn + i, *v.shape))
            want = step(x, dy)
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                other = step(x, dy)
            side.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for a, b, c in zip(want, outs, other):
                assert torch.equal(a, b) and torch.equal(a, c), turn


def test_refusals_on_the_device():
    announce("blocknorm refusals")
    x = inputs(30, 2, 5, 40, torch.bfloat16)
    for bad in (dict(gate=x["gate"].float()), dict(residual=x["residual"][:, :4]), dict(scale=x["scale"][:1]),
                dict(scale=x["scale"].double()), dict(weight=x["weight"].half()), dict(post_weight=x["post_weight"][:, :39])):
        with pytest.raises(ValueError):
            layer.blocknorm(**(x | bad))
    with pytest.raises(TypeError):
        layer.blocknorm(**(x | dict(scale=0.5)))
    got = layer.blocknorm(**x)
    grads = torch.zeros(2, 40, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2, 40, device="cuda")
    with pytest.raises(ValueError):
        layer.blocknorm_backward(x["z"], None, x["z"], x["gate"], layer.pack(x["z"][:, :4]), got[2], got[3], x["post_weight"],
                                 x["scale"], x["weight"], *grads)
    with pytest.raises(ValueError):
        layer.blocknorm_backward(x["z"].float(), None, x["z"], x["gate"], got[4], got[2], got[3], x["post_weight"],
                                 x["scale"], x["weight"], *grads)
