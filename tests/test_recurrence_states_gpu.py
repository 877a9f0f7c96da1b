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


def errors_of_runs(a, add):
    """e_t = a_t e_(t-1) + add_t: what an error at each token has become."""
    e, now = np.zeros_like(add), np.zeros(add.shape[1:])
    for t in range(len(add)):
        now = a[t] * now + add[t]
        e[t] = now
    return e


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,w", [(70000, 3), (5000, 70)])
def test_a_long_sequence_and_its_memory(t, w, dtype):
    """A token's factors a and c are off by some 10 steps of 2^-24, and each has its
    place in a run's product or in a state's step, with up to 4 roundings: E = 14 * 2^-24
    of the size of the state there.  What that has become at a later
    token has faded with it, as the state has: e_t = a_t e_(t-1) + E size_t, and
    backwards alike.  dgate has the errors of dh and of the state before, and E for
    its own products; results are rounded once."""
    announce(f"recurrence {t} x {w} against its memory {dtype}")
    rng = np.random.default_rng(2)
    make = [torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in
            ((1, t, w), (1, t, w), (1, 1, w), (1, t, w), (1, 1, w))]
    gate, x, initial, dh, dlast = make
    gate, x, dh = (1.5 * gate + 1.0).to(dtype), x.to(dtype), (0.1 * dh).to(dtype)
    h, last, saved = layer.recurrence(gate, x, initial)
    got = (h, last, *layer.recurrence_backward(dh, dlast, gate, x, saved, initial))
    wide = [host(v) for v in (gate, x, initial, dh, dlast)]
    f, xs, i0, d, dl = wide
    starts = [[0, t]]
    want = plain.recurrence(f, xs, i0, starts, d, dl)
    size = plain.recurrence(f, np.abs(xs), np.abs(i0), starts, np.abs(d), np.abs(dl))
    a, c = plain.sigmoid(f)[0], plain.sigmoid(-f)[0]
    each, u = 14 * 2.0 ** -24, {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126
    eh = errors_of_runs(a, each * size[0][0])
    flow = size[3][0] / c                                  # |dh|, everything that flows back
    # g_t -> a_t (dy_t + g_t): the error of dh_t is that of a_(t+1) dh_(t+1).
    back = errors_of_runs(np.concatenate([np.zeros((1, w)), a[1:]])[::-1], each * flow[::-1])[::-1]
    prior = np.concatenate([np.abs(i0[0]), size[0][0][:-1]])
    eprior = np.concatenate([np.zeros((1, w)), eh[:-1]])
    slope = a * c
    offs = (eh, eh[-1:], back * (prior + np.abs(xs[0])) * slope + flow * eprior * slope + each * flow * (prior + np.abs(xs[0])) * slope,
            back * c + each * size[3][0], a[:1] * back[:1] + each * size[4][0])
    for g, v, off, what in zip(got, want, offs, ("h", "last", "dgate", "dx", "dinitial")):
        g, v = host(g)[0], v[0]
        lim = off + (u * np.abs(v) + tiny if what in ("h", "dgate", "dx") else 2.0 ** -24 * np.abs(v) + 2.0 ** -126)
        bad = np.abs(g - v) > lim
        assert not bad.any(), (what, int(bad.sum()), float(np.abs(g - v)[bad].max()))
