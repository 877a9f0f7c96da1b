"""Plain 64-bit gated recurrence and its gradients from their definitions, one
token at a time; numpy arrays in and out."""
from __future__ import annotations

import numpy as np


def sigmoid(f):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-f))


def recurrence(gate, x, initial, starts, dh=None, dlast=None):
    """(h, last), and with dh also (dgate, dx, dinitial); starts lists each
    worker's sequences, initial and dlast are [n][count][width] or None."""
    gate, x = gate.astype(np.float64), x.astype(np.float64)
    n, tokens, width = gate.shape
    count = len(starts[0]) - 1
    a, c = sigmoid(gate), sigmoid(-gate)
    zero = np.zeros((n, count, width))
    initial = zero if initial is None else initial.astype(np.float64)
    h, last = np.zeros_like(x), initial.copy()
    prior = np.zeros_like(x)
    for i in range(n):
        for s in range(count):
            state = initial[i, s]
            for t in range(starts[i][s], starts[i][s + 1]):
                prior[i, t] = state
                state = h[i, t] = a[i, t] * state + c[i, t] * x[i, t]
            last[i, s] = state
    if dh is None:
        return h, last
    dlast = zero if dlast is None else dlast.astype(np.float64)
    dgate, dx, dinitial = np.zeros_like(x), np.zeros_like(x), dlast.copy()
    for i in range(n):
        for s in range(count):
            back = dlast[i, s]
            for t in reversed(range(starts[i][s], starts[i][s + 1])):
                d = dh[i, t] + back
                dgate[i, t] = d * (prior[i, t] - x[i, t]) * a[i, t] * c[i, t]
                dx[i, t] = c[i, t] * d
                back = a[i, t] * d
            dinitial[i, s] = back
    return h, last, dgate, dx, dinitial
