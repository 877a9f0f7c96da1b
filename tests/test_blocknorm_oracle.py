"""CPU: the plain norms around a block (oracle/layer.py) against differences,
and the calls' refusals that need no device."""
import numpy as np
import pytest

import paper_2110_04175_amd as rs
from oracle import layer as plain
from paper_2110_04175_amd import layer


def test_a_case_worked_by_hand():
    """z = (3, 4): rms 5 / sqrt(2); gates of 0 halve."""
    z = np.array([3.0, 4.0]).reshape(1, 1, 2)
    s, size, rstd = plain.blocknorm(z, np.zeros_like(z), np.ones_like(z), np.array([[5.0, 10.0]]), np.array([-2.0]), 0.0)
    assert np.allclose(rstd, np.sqrt(2) / 5)
    assert np.allclose(s, 1 - np.sqrt(2) * np.array([3.0, 8.0])) and np.allclose(size, np.sqrt(2) * np.array([3.0, 8.0]))


@pytest.mark.parametrize("gated", [True, False])
def test_gradients_against_differences(gated):
    rng = np.random.default_rng(1)
    n, t, w, eps = 2, 3, 5, 1e-3
    z, gate, r, dy, dsum = (rng.standard_normal((n, t, w)) for _ in range(5))
    post, weight, scale = 1 + 0.1 * rng.standard_normal((n, w)), 1 + 0.1 * rng.standard_normal((n, w)), rng.standard_normal(n)
    if not gated:
        gate = None

    def forward(z, gate, r, post, scale, weight):
        s, _, post_rstd = plain.blocknorm(z, gate, r, post, scale, eps)
        return s, plain.rmsnorm(s, weight, eps), post_rstd

    args = [z, gate, r, post, scale, weight]
    s, (y, rstd), post_rstd = forward(*args)
    ds, dz, dgate, dw, dp, dsc = plain.blocknorm_backward(dy, dsum, z, gate, s, post_rstd, rstd, post, scale, weight)

    def loss(args):
        s, (y, _), _ = forward(*args)
        return np.sum(y * dy) + np.sum(s * dsum)

    for which, g in ((0, dz), (1, dgate), (2, ds), (3, dp), (4, dsc), (5, dw)):
        if args[which] is None:
            assert g is None
            continue
        for at in range(args[which].size):
            step = np.zeros(args[which].size)
            step[at] = 1e-6
            step = step.reshape(args[which].shape)
            up, down = ([v + sign * step if j == which else v for j, v in enumerate(args)] for sign in (1, -1))
            assert abs((loss(up) - loss(down)) / 2e-6 - g.reshape(-1)[at]) < 1e-7


BASE = 1 << 40


def rows(at, n, t, w, type=1):
    return layer.Rows(at, type, t * w, w)


def forward(n=2, t=8, w=200, eps=1e-6, scale=20 * BASE, scale_stride=1, stride=200, post=21 * BASE, weight=22 * BASE,
            saved=True, ygroup=0, sgroup=128, **change):
    x = {"z": rows(BASE, n, t, w), "gate": rows(2 * BASE, n, t, w), "residual": rows(3 * BASE, n, t, w),
         "sum": rows(4 * BASE, n, t, w)}
    x.update(change)
    lib = layer._lib()
    rc = lib.relaysum_blocknorm(n, t, w, x["z"], x["gate"], x["residual"], post, stride, scale, scale_stride, weight, stride,
                                eps, x["sum"], layer._CPacked(5 * BASE, 6 * BASE, ygroup), 7 * BASE, 8 * BASE,
                                layer._CPacked(9 * BASE, 10 * BASE, sgroup) if saved else None, None)
    return rc, lib.relaysum_layer_error().decode()


@pytest.mark.parametrize("text,kw", [
    ("n must be", dict(n=0)), ("width", dict(w=0)), ("width", dict(w=32769)), ("tokens", dict(t=-1)), ("eps", dict(eps=-1.0)),
    ("eps", dict(eps=float("nan"))), ("NULL", dict(z=None)), ("NULL", dict(residual=None)), ("NULL", dict(sum=None)),
    ("NULL", dict(post=None)), ("NULL", dict(weight=None)), ("NULL", dict(scale=None)), ("aligned", dict(scale=BASE + 1)),
    ("stride", dict(scale_stride=-1)), ("stride", dict(stride=-1)), ("z's type", dict(gate=rows(2 * BASE, 2, 8, 200, 0))),
    ("z's type", dict(residual=rows(2 * BASE, 2, 8, 200, 2))), ("z's type", dict(sum=rows(4 * BASE, 2, 8, 200, 2))),
    ("whole rows", dict(ygroup=128)), ("groups of", dict(sgroup=0)), ("share memory", dict(sum=rows(BASE + 2, 2, 8, 200))),
    ("share memory", dict(sum=rows(21 * BASE, 2, 8, 200))),
])
def test_refusals(text, kw):
    rc, said = forward(**kw)
    assert rc == rs.RELAYSUM_ERR_INVALID_ARG and text in said, said


@pytest.mark.parametrize("at", [1, 2, 3])
def test_the_sum_in_place(at):
    rc, said = forward(sum=rows(at * BASE, 2, 8, 200))
    assert rc != 0 and "share" not in said


def test_refused_backward():
    lib = layer._lib()
    n, t, w = 2, 50, 200
    a = {name: rows((i + 1) * BASE, n, t, w) for i, name in enumerate(("dy", "dsum", "z", "gate", "dz", "dgate", "ds"))}
    g = {name: layer.Rows((30 + i) * BASE, 0, w, 0) for i, name in enumerate(("post", "scale", "weight"))}

    def call(size=1 << 30, **change):
        x = a | g | change
        rc = lib.relaysum_blocknorm_backward(n, t, w, x["dy"], x["dsum"], x["z"], x["gate"], layer._CPacked(10 * BASE, 11 * BASE, 128),
                                             12 * BASE, 13 * BASE, 14 * BASE, w, 15 * BASE, 1, 16 * BASE, w, x["dz"], x["dgate"],
                                             x["ds"], x["post"], x["scale"], x["weight"], 40 * BASE, size, None)
        return rc, lib.relaysum_layer_error().decode()

    for name in ("dy", "z", "dz", "ds", "post", "scale", "weight"):
        rc, said = call(**{name: None})
        assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "NULL" in said, (name, said)
    for kw, text in ((dict(gate=None), "come together"), (dict(dgate=None), "come together"), (dict(size=8), "workspace"),
                     (dict(dy=rows(BASE, n, t, w, 0)), "z's type"), (dict(dz=rows(5 * BASE, n, t, w, 2)), "z's type"),
                     (dict(post=layer.Rows(30 * BASE, 1, w, 0)), "float"), (dict(dz=rows(7 * BASE, n, t, w)), "share memory"),
                     (dict(scale=layer.Rows(30 * BASE, 0, 1, 0)), "share memory")):
        rc, said = call(**kw)
        assert rc == rs.RELAYSUM_ERR_INVALID_ARG and text in said, (kw, said)
    rc, said = call(dz=rows(3 * BASE, n, t, w), ds=rows(1 * BASE, n, t, w), dgate=rows(4 * BASE, n, t, w))   # in place
    assert rc != 0 and "share" not in said
    assert lib.relaysum_blocknorm_workspace(0, 1, 1) == -1 and lib.relaysum_blocknorm_workspace(2, 1, 100) == 0
