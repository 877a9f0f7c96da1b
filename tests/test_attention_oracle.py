"""CPU: the plain attention (oracle/attention.py) is pinned against a
hand-worked case and differences, and the calls' refusals that need no
device."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2110_04175_amd as rs
from oracle import attention as plain
from paper_2110_04175_amd import layer


def test_a_case_worked_by_hand():
    """Two keys with scores 0 and log 3: weights 1/4 and 3/4."""
    q = np.ones((1, 1, 1, 1))
    k = np.array([0.0, np.log(3.0)]).reshape(1, 2, 1, 1)
    v = np.array([4.0, 8.0]).reshape(1, 2, 1, 1)
    out, lse, size = plain.attention(q, k, v, plain.default_ranges(1, 1, 2, True), 1.0)
    assert np.allclose(out, 7.0) and np.allclose(lse, np.log(4.0)) and np.allclose(size, 7.0)


def test_ranges():
    r = plain.ranges_of([[0, 2, 2, 3]], 5, [[0, 4, 5, 6]], 6, True)
    assert r.tolist() == [[[0, 3], [0, 4], [5, 6], [0, 0], [0, 0]]]
    r = plain.ranges_of([[0, 3]], 3, [[0, 1]], 1, True)
    assert r.tolist() == [[[0, 0], [0, 0], [0, 1]]]
    assert plain.default_ranges(1, 2, 3, True).tolist() == [[[0, 2], [0, 3]]]


def test_heads_share_keys():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((1, 3, 4, 5)), rng.standard_normal((1, 6, 2, 5)), rng.standard_normal((1, 6, 2, 5))
    r = plain.default_ranges(1, 3, 6, True)
    out = plain.attention(q, k, v, r, 0.5)[0]
    for h in range(4):
        one = plain.attention(q[:, :, h:h + 1], k[:, :, h // 2:h // 2 + 1], v[:, :, h // 2:h // 2 + 1], r, 0.5)[0]
        assert np.allclose(one[:, :, 0], out[:, :, h])


@pytest.mark.parametrize("seed", range(3))
def test_gradients_against_differences(seed):
    rng = np.random.default_rng(seed)
    n, t, keys, h, kv, w = 2, 4, 5, 4, 2, 3
    q, do = rng.standard_normal((n, t, h, w)), rng.standard_normal((n, t, h, w))
    k, v = rng.standard_normal((n, keys, kv, w)), rng.standard_normal((n, keys, kv, w))
    r = np.sort(rng.integers(0, keys + 1, (n, t, 2)), 2)
    grads = plain.attention(q, k, v, r, 0.7, do)[3]
    for x, g in zip((q, k, v), grads):
        for at in rng.choice(x.size, 20):
            one = np.zeros(x.size)
            one[at] = 1e-6
            step = one.reshape(x.shape)
            moved = []
            for sign in (1, -1):
                args = [y + sign * step if y is x else y for y in (q, k, v)]
                moved.append(np.sum(plain.attention(*args, r, 0.7)[0] * do))
            assert abs((moved[0] - moved[1]) / 2e-6 - g.reshape(-1)[at]) < 1e-7


# ---- refusals: addresses that are no device memory; every call fails, what is
# wrong with the arguments before anything is asked about them.

BASE = 1 << 40


def heads(at, n, rows, h, w, type=1, ws=None, rs_=None, hs=None):
    return layer.Heads(at, type, rows * h * w if ws is None else ws, h * w if rs_ is None else rs_, w if hs is None else hs)


def forward(n=2, t=8, keys=8, h=4, kv=2, w=32, scale=0.1, ranges=None, stride=0, lse=None, ws=None, size=1 << 30, **change):
    lib = layer._lib()
    x = {"q": heads(BASE, n, t, h, w), "k": heads(2 * BASE, n, keys, kv, w), "v": heads(3 * BASE, n, keys, kv, w),
         "out": heads(4 * BASE, n, t, h, w)}
    x.update(change)
    rc = lib.relaysum_attention(n, t, keys, h, kv, w, x["q"], x["k"], x["v"], ranges, stride, 1, scale, x["out"], lse,
                                ws, size, None)
    return rc, lib.relaysum_layer_error().decode()


def refused(text, **kw):
    rc, said = forward(**kw)
    assert rc == rs.RELAYSUM_ERR_INVALID_ARG and text in said, said


def test_refused_sizes():
    refused("multiple of kv_heads", h=3)
    refused("multiple of kv_heads", h=0)
    refused("multiple of kv_heads", kv=0)
    refused("multiple of kv_heads", kv=-2)
    refused("width", w=0)
    refused("width", w=257)
    refused("n must be", n=0)
    refused("tokens", t=-1)
    refused("keys", keys=-1)
    refused("2^30", keys=(1 << 30) + 1)
    refused("2^30", t=1 << 29)
    for scale in (0.0, -0.5, float("nan"), float("inf")):
        refused("scale", scale=scale)


def test_refused_arrays():
    refused("must not be NULL", q=None)
    refused("must not be NULL", v=None)
    refused("must not be NULL", k=heads(0, 2, 8, 2, 32))
    refused("unknown type", q=heads(BASE, 2, 8, 4, 32, type=3))
    refused("not of q's type", v=heads(BASE, 2, 8, 2, 32, type=2))
    refused("aligned", q=heads(BASE + 1, 2, 8, 4, 32))
    refused("negative", k=heads(BASE, 2, 8, 2, 32, rs_=-64))
    refused("2^44", k=heads(BASE, 2, 8, 2, 32, ws=1 << 44))
    refused("rows overlap", out=heads(4 * BASE, 2, 8, 4, 32, hs=31))
    refused("rows overlap", out=heads(4 * BASE, 2, 8, 4, 32, rs_=0))
    refused("rows overlap", out=heads(4 * BASE, 2, 8, 4, 32, ws=64))
    refused("share memory", out=heads(BASE + 64, 2, 8, 4, 32))
    refused("share memory", lse=2 * BASE)
    refused("ranges_stride", ranges=5 * BASE, stride=7)
    refused("aligned", ranges=5 * BASE + 4, stride=8)
    refused("aligned", lse=5 * BASE + 2)


def test_outputs_beside_inputs():
    """Parts of one array's rows are apart, heads of one row too."""
    rc, said = forward(q=heads(BASE, 2, 8, 4, 32, ws=8 * 256, rs_=256), out=heads(BASE + 256, 2, 8, 4, 32, ws=8 * 256, rs_=256))
    assert rc != 0 and "share" not in said
    refused("share memory", q=heads(BASE, 2, 8, 4, 32, ws=8 * 256, rs_=256),
            out=heads(BASE + 254, 2, 8, 4, 32, ws=8 * 256, rs_=256))
    rc, said = forward(q=heads(BASE, 2, 8, 4, 32, ws=8 * 256, rs_=256, hs=64), out=heads(BASE + 64, 2, 8, 4, 32, ws=8 * 256, rs_=256, hs=64))
    assert rc != 0 and "share" not in said


def test_workspaces():
    lib = layer._lib()
    size = lib.relaysum_attention_workspace(1, 1, 100000, 8, 1, 128)
    assert size > 0 and size % 4 == 0
    rc, said = forward(n=1, t=1, keys=100000, h=8, kv=1, w=128, ws=6 * BASE, size=size - 1)
    assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "workspace" in said
    assert 0 < lib.relaysum_attention_workspace(64, 2048, 2048, 16, 16, 64) <= 1 << 20
    assert lib.relaysum_attention_workspace(1, 1, 1, 3, 2, 64) == -1
    assert lib.relaysum_attention_backward_workspace(1, 1, 1, 3, 2, 64, 0) == -1
    assert lib.relaysum_attention_backward_workspace(1, 1, 1, 2, 2, 64, 3) == -1
    for t in (0, 1, 2):
        assert lib.relaysum_attention_backward_workspace(2, 100, 100, 4, 2, 64, t) >= 2 * 100 * 4 * 4


def test_refused_backward():
    lib = layer._lib()
    n, t, h, kv, w = 2, 8, 4, 2, 32
    a = [heads((i + 1) * BASE, n, t, h if i in (0, 1, 4, 5) else kv, w) for i in range(8)]

    def call(x, size=1 << 30):
        rc = lib.relaysum_attention_backward(n, t, t, h, kv, w, *x[:5], 20 * BASE, None, 0, 1, 0.1, *x[5:], 21 * BASE, size, None)
        return rc, lib.relaysum_layer_error().decode()

    rc, said = call(a, 15)
    assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "workspace" in said
    for i in range(8):
        rc, said = call([None if j == i else x for j, x in enumerate(a)])
        assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "NULL" in said
    rc, said = call([heads(6 * BASE, n, t, kv, w) if j == 6 else x for j, x in enumerate(a)])   # dk over dq
    assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "share memory" in said


def test_refused_ranges():
    lib = layer._lib()

    def call(n=2, t=8, keys=8, count=3, stride=4, kstride=4, starts=BASE, out=2 * BASE, rstride=8):
        rc = lib.relaysum_attention_ranges(n, t, keys, count, starts, stride, 3 * BASE, kstride, 1, out, rstride, None)
        return rc, lib.relaysum_layer_error().decode()

    for text, kw in (("count", dict(count=0)), ("negative", dict(stride=-1)), ("NULL", dict(starts=None)),
                     ("NULL", dict(out=None)), ("ranges_stride", dict(rstride=4)),
                     ("share memory", dict(out=BASE)), ("tokens", dict(t=-1))):
        rc, said = call(**kw)
        assert rc == rs.RELAYSUM_ERR_INVALID_ARG and text in said, (text, said)


def test_python_refusals_without_a_device():
    x = torch.zeros(1, 2, 1, 4)
    with pytest.raises(TypeError):
        layer.attention(x, x, x)
    with pytest.raises(ValueError):
        layer.attention_ranges(torch.zeros(2, dtype=torch.int32), 4, key_starts=torch.zeros(2, dtype=torch.int32))
    assert ctypes.sizeof(layer.Heads) == 40
