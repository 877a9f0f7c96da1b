"""CPU: the plain recurrence (oracle/recurrence.py) is pinned against a
hand-worked case and differences, and the calls' refusals that need no
device."""
import numpy as np
import pytest

import paper_2110_04175_amd as rs
from oracle import recurrence as plain
from paper_2110_04175_amd import layer


def test_a_case_worked_by_hand():
    """Gates of 0 keep half: from 8, with inputs 4 and 2, to 6 and 4; from 1
    with 3 to 2; a sequence of nothing keeps its 5."""
    gate = np.zeros((1, 4, 1))
    x = np.array([4.0, 2.0, 3.0, 9.0]).reshape(1, 4, 1)
    initial = np.array([8.0, 5.0, 1.0]).reshape(1, 3, 1)
    h, last = plain.recurrence(gate, x, initial, [[0, 2, 2, 3]])
    assert h.ravel().tolist() == [6.0, 4.0, 2.0, 0.0]
    assert last.ravel().tolist() == [4.0, 5.0, 2.0]
    out = plain.recurrence(gate, x, initial, [[0, 2, 2, 3]], np.ones((1, 4, 1)), np.ones((1, 3, 1)))
    # dh: 1 + 1 = 2 at the end, 1 + 2 / 2 = 2 before it, half of that for the state.
    assert out[3].ravel().tolist() == [1.0, 1.0, 1.0, 0.0]
    assert out[4].ravel().tolist() == [1.0, 1.0, 1.0]
    assert out[2].ravel().tolist() == [2 * (8 - 4) / 4, 2 * (6 - 2) / 4, 2 * (1 - 3) / 4, 0.0]


@pytest.mark.parametrize("seed", range(3))
def test_gradients_against_differences(seed):
    rng = np.random.default_rng(seed)
    n, t, w, count = 2, 7, 3, 3
    starts = [sorted(rng.integers(0, t + 1, count + 1).tolist()) for _ in range(n)]
    gate, x, dh = (rng.standard_normal((n, t, w)) for _ in range(3))
    initial, dlast = (rng.standard_normal((n, count, w)) for _ in range(2))
    grads = plain.recurrence(gate, x, initial, starts, dh, dlast)[2:]

    def loss(*args):
        h, last = plain.recurrence(*args, starts)
        return np.sum(h * dh) + np.sum(last * dlast)

    for which, g in enumerate(grads):
        args = [gate, x, initial]
        for at in rng.choice(args[which].size, 12):
            step = np.zeros(args[which].size)
            step[at] = 1e-6
            step = step.reshape(args[which].shape)
            up, down = ([v + sign * step if j == which else v for j, v in enumerate(args)] for sign in (1, -1))
            assert abs((loss(*up) - loss(*down)) / 2e-6 - g.reshape(-1)[at]) < 1e-8


BASE = 1 << 40


def rows(at, n, t, w, type=1):
    return layer.Rows(at, type, t * w, w)


def forward(n=2, t=200, w=32, count=3, starts=9 * BASE, stride=4, ws=8 * BASE, size=1 << 30, saved=None, **change):
    x = {"gate": rows(BASE, n, t, w), "x": rows(2 * BASE, n, t, w), "initial": None, "h": rows(3 * BASE, n, t, w),
         "last": None}
    x.update(change)
    lib = layer._lib()
    rc = lib.relaysum_recurrence(n, t, w, count, starts, stride, x["gate"], x["x"], x["initial"], x["h"], x["last"],
                                 saved, ws, size, None)
    return rc, lib.relaysum_layer_error().decode()


@pytest.mark.parametrize("text,kw", [
    ("n must be", dict(n=0)), ("width", dict(w=0)), ("width", dict(w=32769)), ("tokens", dict(t=-1)),
    ("tokens", dict(t=(1 << 30) + 1)), ("count", dict(count=0)), ("one sequence", dict(starts=None)),
    ("starts_stride", dict(stride=-1)), ("aligned", dict(starts=9 * BASE + 2)),
    ("NULL", dict(gate=None)), ("NULL", dict(x=None)), ("NULL", dict(h=None)),
    ("one type", dict(x=rows(2 * BASE, 2, 200, 32, 0))), ("unknown type", dict(gate=rows(BASE, 2, 200, 32, 7))),
    ("type float", dict(initial=rows(5 * BASE, 2, 3, 32))), ("type float", dict(last=rows(5 * BASE, 2, 3, 32))),
    ("share memory", dict(h=rows(BASE, 2, 200, 32))), ("share memory", dict(last=rows(3 * BASE, 2, 3, 32, 0))),
    ("share memory", dict(saved=3 * BASE)), ("workspace", dict(t=1000, size=100)),
    ("NULL", dict(t=1000, ws=None)),
    ("too large", dict(n=1 << 24, t=1, w=512, count=1)),
])
def test_refusals(text, kw):
    rc, said = forward(**kw)
    assert rc == rs.RELAYSUM_ERR_INVALID_ARG and text in said, said


def test_refused_backward():
    lib = layer._lib()
    n, t, w, count = 2, 1000, 32, 1
    a = [rows((i + 1) * BASE, n, t, w) for i in range(5)]   # dh, gate, x, dgate, dx

    def call(x, saved=7 * BASE, size=1 << 30):
        rc = lib.relaysum_recurrence_backward(n, t, w, count, None, 0, x[0], None, x[1], x[2], None, saved, x[3], x[4],
                                              None, 8 * BASE, size, None)
        return rc, lib.relaysum_layer_error().decode()

    for i in range(5):
        rc, said = call([None if j == i else x for j, x in enumerate(a)])
        assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "NULL" in said
        rc, said = call([rows((i + 1) * BASE, n, t, w, 2) if j == i else x for j, x in enumerate(a)])
        assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "one type" in said
    for kw, text in ((dict(saved=None), "NULL"), (dict(size=8), "workspace"), (dict(saved=4 * BASE), "share")):
        rc, said = call(a, **kw)
        assert rc == rs.RELAYSUM_ERR_INVALID_ARG and text in said


def test_sizes():
    lib = layer._lib()
    assert [lib.relaysum_recurrence_chunks(t) for t in (0, 1, 64, 65, -1)] == [1, 1, 1, 2, -1]
    assert layer.CHUNK == 64
    # Parts where there are few channels for many tokens.
    assert lib.relaysum_recurrence_workspace(3, 64, 100) == 0
    assert lib.relaysum_recurrence_workspace(3, 1000, 100) > 0
    assert lib.relaysum_recurrence_workspace(16, 2048, 1024) == 0
    assert lib.relaysum_recurrence_workspace(0, 65, 100) == -1
