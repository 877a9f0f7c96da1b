"""GPU: the recurrence's 32-bit results, whatever type its rows have, and a long
sequence against the memory that it has."""
import sys

import numpy as np
import pytest
import torch

from oracle import recurrence as plain
from paper_2110_04175_amd import layer

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


def host(t):
    return t.double().cpu().numpy()


def states(gate, x, initial, dh, dlast, starts):
    """(last, dinitial) one token at a time, in the arrays' own precision."""
    one = gate.dtype.type(1)
    a, c = one / (one + np.exp(-gate)), one / (one + np.exp(gate))
    last, first = initial.copy(), dlast.copy()
    for i in range(gate.shape[0]):
        for s in range(initial.shape[1]):
            b, e = starts[s], starts[s + 1]
            for t in range(b, e):
                last[i, s] = a[i, t] * last[i, s] + c[i, t] * x[i, t]
            for t in reversed(range(b, e)):
                first[i, s] = a[i, t] * (first[i, s] + dh[i, t])
    return last, first


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("spread", [1.0, 2.0, 3.0])
def test_states_are_as_near_as_floats(spread, dtype):
    """last and dinitial are floats, also of rows in 16 bits, and are as near to 64
    bits as the definition in floats, one token after the other.  A token rounds
    a there four times (the exponential, the sum, the quotient, the product with the
    state) and c as often, and the sum; here as often, and the products
    of a run of 8 tokens once more.  Twice the roundings at most are 2^0.5 of the distance,
    as they are independent; 2 is allowed."""
    announce(f"recurrence states {spread} {dtype}")
    rng = np.random.default_rng(1)
    starts = [0, 1, 4, 20, 70, 70, 400, 1100, 1800]
    n, t, w, count = 2, 1800, 512, len(starts) - 1
    make = [torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in
            ((n, t, w), (n, t, w), (n, count, w), (n, t, w), (n, count, w), (n, 1, w))]
    gate, x, initial, dh, dlast, keep = make
    # Channels that keep between a token and some thousand.
    gate, x, dh = (gate + spread * keep.abs()).to(dtype), x.to(dtype), (0.01 * dh).to(dtype)
    dlast *= 0.01
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    h, last, saved = layer.recurrence(gate, x, initial, st)
    dinitial = layer.recurrence_backward(dh, dlast, gate, x, saved, initial, st)[2]
    wide = [host(v) for v in (gate, x, initial, dh, dlast)]
    want = states(*wide, starts)
    narrow = states(*(v.astype(np.float32) for v in wide), starts)
    for got, a, b, what in zip((last, dinitial), want, narrow, ("last", "dinitial")):
        size = np.linalg.norm(a)
        off, plain_off = np.linalg.norm(host(got) - a) / size, np.linalg.norm(b.astype(np.float64) - a) / size
        announce(f"{what}: {off:.2e}, in floats {plain_off:.2e}")
        assert off <= 2 * plain_off, (what, off, plain_off)
