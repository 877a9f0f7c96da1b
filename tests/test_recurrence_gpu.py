"""GPU: the gated recurrence and its gradients against the plain 64-bit
implementation (oracle/recurrence.py).

Tolerances.  A gate's a and c = 1 - a are off by some 8 steps of 2^-24 (two
exponentials' and reciprocals' units, the sum, the product), and in 16-bit
types by |gate| * 2^-23 more from the exponent's rounding.  h_t is a weighted
mean of what came before: of x and the initial state with weights c a a a ...
Every factor and every step of the sum adds a rounding, for as long as the
product of a's has not faded; a bound that holds for any gates is steps * E of
the mean of |x| with the same weights, E the error of one factor and 2^-24 for
its use.  Sizes are computed by the oracle itself from |x|, |initial|, and in
the gradients from |dh|, |dlast| and |h| + |x|; `steps` is the longest sequence.
Runs of tokens compose by products of a's, which are off by as much."""
import sys

import numpy as np
import pytest
import torch

from oracle import recurrence as plain
from paper_2110_04175_amd import layer

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


def host(t):
    return None if t is None else t.double().cpu().numpy()


def normal(seed, *shape, std=1.0, mean=0.0, dtype=torch.float32):
    g = np.random.default_rng(seed).standard_normal(shape) * std + mean
    return torch.from_numpy(g.astype(np.float32)).cuda().to(dtype)


def inputs(seed, n, t, w, count, dtype):
    return (normal(seed, n, t, w, std=1.5, mean=1.0, dtype=dtype), normal(seed + 1, n, t, w, dtype=dtype),
            normal(seed + 2, n, count, w), normal(seed + 3, n, t, w, std=0.1, dtype=dtype),
            normal(seed + 4, n, count, w, std=0.1))


def finite(v):
    return None if v is None else np.where(np.isfinite(v), v, 0.0)


def bounds(gate, x, initial, starts, dh, dlast, dtype):
    """[(value, how far off)] of h, last, dgate, dx, dinitial."""
    gate, x, dh = finite(gate), finite(x), finite(dh)
    want = plain.recurrence(gate, x, initial, starts, dh, dlast)
    size = plain.recurrence(gate, np.abs(x), None if initial is None else np.abs(initial), starts, np.abs(dh),
                            None if dlast is None else np.abs(dlast))
    a, c = plain.sigmoid(gate), plain.sigmoid(-gate)
    n, t, w = x.shape
    steps = max(max(s[j + 1] - s[j] for j in range(len(s) - 1)) for s in starts)
    one = (10 + (np.abs(gate).max(initial=0) if dtype != torch.float32 else 0)) * ULP
    e = (steps + 8) * one
    u, tiny = ROUND[dtype], TINY[dtype]
    # |h_(t-1)| + |x|, times what flows back.
    flow = np.divide(size[3], c, out=np.zeros_like(c), where=c > 0)
    prior = np.zeros_like(x)
    for i in range(n):
        for j in range(len(starts[i]) - 1):
            b, f = starts[i][j], starts[i][j + 1]
            if f > b:
                prior[i, b] = 0 if initial is None else np.abs(initial[i, j])
                prior[i, b + 1:f] = size[0][i, b:f - 1]
    gsize = flow * (prior + np.abs(x)) * a * c
    return [(want[0], e * size[0] + u * np.abs(want[0]) + tiny), (want[1], e * size[1] + ULP * np.abs(want[1]) + 2.0 ** -126),
            (want[2], 3 * e * gsize + u * np.abs(want[2]) + tiny), (want[3], 2 * e * size[3] + u * np.abs(want[3]) + tiny),
            (want[4], 2 * e * size[4] + ULP * np.abs(want[4]) + 2.0 ** -126)]


NAMES = ("h", "last", "dgate", "dx", "dinitial")


def near(got, want, off, what):
    got = host(got)
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), what
    bad = np.abs(got - want) > off
    assert not bad.any(), (what, np.abs(got - want)[bad].max(), int(bad.sum()), np.argwhere(bad)[:4].tolist())


def run(gate, x, initial, starts, dh, dlast):
    h, last, saved = layer.recurrence(gate, x, initial, starts)
    return (h, last, *layer.recurrence_backward(dh, dlast, gate, x, saved, initial, starts))


def check(gate, x, initial, starts, dh, dlast):
    """starts: a list for each worker, or None."""
    n, t, w = gate.shape
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    got = run(gate, x, initial, st, dh, dlast)
    lists = [[0, t]] * n if starts is None else starts
    found = bounds(host(gate), host(x), host(initial), lists, host(dh), host(dlast), gate.dtype)
    for g, (want, off), what in zip(got, found, NAMES):
        near(g, want, off, what)
    assert torch.equal(layer.recurrence(gate, x, initial, st, keep=False)[0], got[0])
    return got


SHAPES = [(1, 1, 1), (16, 1, 96), (2, 7, 5), (1, 64, 256), (3, 65, 257), (2, 63, 130), (1, 200, 1001), (2, 129, 33),
          (300, 3, 17), (1, 1500, 8)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_one_sequence(shape, dtype):
    announce(f"recurrence {shape} {dtype}")
    n, t, w = shape
    gate, x, initial, dh, dlast = inputs(1, n, t, w, 1, dtype)
    check(gate, x, initial, None, dh, dlast)
    check(gate, x, None, None, dh, None)


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_sequences(dtype):
    """Sequences of no, one and many tokens, starts on and off a chunk's edge,
    other ones for each worker, rows in none that hold NaN."""
    announce(f"recurrence packed {dtype}")
    n, t, w = 3, 300, 40
    starts = [[0, 0, 1, 2, 64, 64, 128, 270], [5, 60, 130, 130, 131, 192, 256, 300], [0, 0, 0, 0, 0, 0, 64, 65]]
    gate, x, initial, dh, dlast = inputs(2, n, t, w, 7, dtype)
    for i, s in enumerate(starts):
        for v in (gate, x, dh):
            v[i, :s[0]] = float("nan")
            v[i, s[-1]:] = float("nan")
    got = check(gate, x, initial, starts, dh, dlast)
    for i, s in enumerate(starts):
        for v in (got[0], got[2], got[3]):
            assert (v[i, :s[0]] == 0).all() and (v[i, s[-1]:] == 0).all()
    check(gate, x, None, starts, dh, None)


@pytest.mark.parametrize("seed", range(6))
def test_random_sequences(seed):
    rng = np.random.default_rng(seed)
    n, t, w = int(rng.integers(1, 4)), int(rng.integers(1, 700)), int(rng.integers(1, 300))
    count = int(rng.integers(1, 20))
    starts = [sorted(rng.integers(0, t + 1, count + 1).tolist()) for _ in range(n)]
    dtype = TYPES[seed % 3]
    announce(f"recurrence random n={n} t={t} w={w} count={count} {dtype}")
    check(*inputs(seed, n, t, w, count, dtype)[:3], starts, *inputs(seed, n, t, w, count, dtype)[3:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count", [7, 63, 64, 200])
def test_sequences_in_parts_of_tokens(count, dtype):
    """Few channels and many tokens, which are split: sequences that begin and end
    within parts, at their edges (512 tokens) and over several of them, fewer and
    more than a wave's lanes, some empty, rows in none that hold NaN."""
    announce(f"recurrence in parts count={count} {dtype}")
    n, t, w = 2, 3000, 70
    rng = np.random.default_rng(count)
    starts = [sorted(rng.integers(0, t - 20, count + 1).tolist()) for _ in range(n)]
    starts[0][1:4] = sorted([512, 512, 1024])
    starts[0] = sorted(starts[0])
    starts[1][0] = 0
    gate, x, initial, dh, dlast = inputs(16, n, t, w, count, dtype)
    for i, s in enumerate(starts):
        for v in (gate, x, dh):
            v[i, :s[0]] = float("nan")
            v[i, s[-1]:] = float("nan")
    got = check(gate, x, initial, starts, dh, dlast)
    for i, s in enumerate(starts):
        for v in (got[0], got[2], got[3]):
            assert (v[i, :s[0]] == 0).all() and (v[i, s[-1]:] == 0).all()


def test_shared_starts():
    announce("recurrence shared starts")
    gate, x, initial, dh, dlast = inputs(3, 3, 100, 50, 2, torch.bfloat16)
    one = torch.tensor([0, 30, 90], dtype=torch.int32, device="cuda")
    a = run(gate, x, initial, one, dh, dlast)
    b = run(gate, x, initial, one.expand(3, 3), dh, dlast)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_a_sequence_in_parts():
    """Given back as initial, last lets a sequence go on; token by token it is
    what it was at once."""
    announce("recurrence token by token")
    gate, x, initial, _, _ = inputs(4, 2, 70, 100, 1, torch.float32)
    h, last, _ = layer.recurrence(gate, x, initial)
    state = initial
    for t in range(70):
        one, state, saved = layer.recurrence(gate[:, t:t + 1], x[:, t:t + 1], state, keep=False)
        assert saved is None
        assert torch.allclose(one[:, 0], h[:, t], rtol=2e-5, atol=1e-6)
    assert torch.allclose(state, last, rtol=2e-5, atol=1e-6)


def test_a_batch_of_single_tokens():
    announce("recurrence of many single tokens")
    n, w, count = 2, 70, 150
    gate, x, initial, dh, dlast = inputs(5, n, count, w, count, torch.float16)
    check(gate, x, initial, [list(range(count + 1))] * n, dh, dlast)


@pytest.mark.parametrize("dtype", TYPES)
def test_gates_at_both_ends(dtype):
    """Gates that keep or replace everything, infinities among them."""
    announce(f"recurrence extreme gates {dtype}")
    n, t, w = 1, 150, 64
    gate, x, initial, dh, dlast = inputs(6, n, t, w, 1, dtype)
    gate[:, ::3] = 20.0
    gate[:, 1::5] = -20.0
    check(gate, x, initial, None, dh, dlast)
    gate[:, 20:40] = float("inf")
    gate[:, 60:62] = -float("inf")
    h, last, dgate, dx, dinitial = run(gate, x, initial, None, dh, dlast)
    for v in (h, last, dgate, dx, dinitial):
        assert torch.isfinite(v).all()
    # Every state is off by the bound for 150 steps of values within the largest
    # input, however runs of tokens were composed.
    most = max(float(x.abs().max()), float(initial.abs().max()))
    assert ((h[:, 20:40] - h[:, 19:20]).abs().double() <=
            2 * 158 * 10 * ULP * most + 2 * ROUND[dtype] * h[:, 20:40].abs().double()).all()
    # c is 1 up to the steps that the top of this file counts.
    assert ((h[:, 60:62] - x[:, 60:62]).abs().double() <= (10 * ULP + ROUND[dtype]) * x[:, 60:62].abs().double() + 2.0 ** -120).all()
    assert (dgate[:, 20:40] == 0).all() and (dx[:, 20:40] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_seen_has_no_part(bad):
    """NaN in a sequence goes on to its end, forward, and to its start,
    backward; it reaches no other sequence and no other channel."""
    announce(f"recurrence {bad}")
    starts = [[0, 50, 130, 200]]
    gate, x, initial, dh, dlast = inputs(7, 1, 200, 30, 3, torch.float32)
    good = check(gate, x, initial, starts, dh, dlast)
    x[0, 100, 5] = bad
    dh[0, 110, 7] = bad
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    got = run(gate, x, initial, st, dh, dlast)
    other = [c for c in range(30) if c not in (5, 7)]
    for g, want in zip(got, good):
        rows = g.shape[1]
        assert torch.equal(g[:, :, other], want[:, :, other])
        for part in ((slice(0, 50), slice(130, 200)) if rows == 200 else (slice(0, 1), slice(2, 3))):
            assert torch.equal(g[:, part], want[:, part])
    assert torch.equal(got[0][0, 50:100, 5], good[0][0, 50:100, 5]) and not torch.isfinite(got[0][0, 100:130, 5]).any()
    assert torch.equal(got[3][0, 111:130, 7], good[3][0, 111:130, 7]) and not torch.isfinite(got[3][0, 50:111, 7]).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_strides(dtype):
    """Parts of wider rows that start anywhere, workers inside tokens,
    broadcast inputs."""
    announce(f"recurrence strides {dtype}")
    n, t, w = 3, 90, 37
    gate, x, initial, dh, dlast = inputs(8, n, t, w, 1, dtype)
    good = check(gate, x, initial, None, dh, dlast)
    wide = normal(9, n, t, 2 * w + 3, dtype=dtype)
    g2, x2 = wide[:, :, 1:1 + w], wide[:, :, 2 + w:2 + 2 * w]
    g2.copy_(gate)
    x2.copy_(x)
    d2 = dh.transpose(0, 1).contiguous().transpose(0, 1)
    states = torch.zeros(n, 2 * w + 1, device="cuda")
    i2 = states[:, None, w:2 * w]
    i2.copy_(initial)
    got = run(g2, x2, i2, None, d2, dlast)
    assert all(torch.equal(p, q) for p, q in zip(got, good))
    check(gate[:1].expand(n, t, w), x[:, :1].expand(n, t, w), initial, None, dh, dlast)


def test_far_rows():
    announce("recurrence far rows")
    far = torch.empty(1, 70, 1 << 26, dtype=torch.bfloat16, device="cuda")
    gate, x, initial, dh, dlast = inputs(10, 1, 70, 40, 1, torch.bfloat16)
    far[:, :, -40:] = gate
    far[:, :, 3:43] = x
    a = run(gate, x, initial, None, dh, dlast)
    b = run(far[:, :, -40:], far[:, :, 3:43], initial, None, dh, dlast)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_no_tokens():
    announce("recurrence of nothing")
    gate, x, initial, dh, dlast = inputs(11, 2, 0, 30, 1, torch.float16)
    got = run(gate, x, initial, None, dh, dlast)
    assert got[0].shape == (2, 0, 30) and torch.equal(got[1], initial) and torch.equal(got[4], dlast)
    assert (run(gate, x, None, None, dh, None)[1] == 0).all()
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    three = normal(12, 2, 3, 30)
    assert torch.equal(run(gate, x, three, st, dh, None)[1], three)


def test_a_long_sequence():
    """70,000 tokens whose gates fade within some hundred."""
    announce("recurrence long")
    gate, x, initial, dh, dlast = inputs(13, 1, 70000, 3, 1, torch.float32)
    check(gate, x, initial, None, dh, dlast)


def test_equal_bits_and_streams():
    announce("recurrence twice and on a stream")
    args = inputs(14, 4, 1000, 300, 1, torch.bfloat16)
    gate, x, initial, dh, dlast = args
    a = run(gate, x, initial, None, dh, dlast)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = run(gate, x, initial, None, dh, dlast)
    s.synchronize()
    for _ in range(3):
        c = run(gate, x, initial, None, dh, dlast)
        assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(a, b, c))


def test_two_captured_graphs():
    announce("recurrence in graphs")
    made = []
    for seed, t, starts in ((20, 500, [0, 100, 400, 500]), (30, 90, [0, 64, 64, 80])):
        args = inputs(seed, 2, t, 70, 3, torch.float16)
        st = torch.tensor(starts, dtype=torch.int32, device="cuda")
        run(*args[:3], st, *args[3:])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = run(*args[:3], st, *args[3:])
        made.append((args, st, g, outs))
    for turn in range(3):
        for args, st, g, outs in made:
            for i, v in enumerate(args):
                v.copy_(normal(100 + 10 * turn + i, *v.shape))
            want = run(*args[:3], st, *args[3:])
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(want, outs)), turn


def test_refusals_on_the_device():
    announce("recurrence refusals")
    gate, x, initial, dh, dlast = inputs(15, 2, 10, 30, 1, torch.float16)
    for bad in (dict(x=x.float()), dict(x=x[:, :9]), dict(initial=initial.half()), dict(initial=initial[:, :, :29]),
                dict(starts=torch.tensor([0, 10], device="cuda")),
                dict(starts=torch.tensor([[0, 10]], dtype=torch.int32, device="cuda")),
                dict(starts=torch.tensor([0], dtype=torch.int32, device="cuda"))):
        args = dict(gate=gate, x=x, initial=initial, starts=None) | bad
        with pytest.raises(ValueError):
            layer.recurrence(**args)
    with pytest.raises(TypeError):
        layer.recurrence(gate, x.cpu())
    h, last, saved = layer.recurrence(gate, x, initial)
    with pytest.raises(ValueError):
        layer.recurrence_backward(dh, dlast, gate, x, saved[:, :, :20], initial)
    with pytest.raises(ValueError):
        layer.recurrence_backward(dh.float(), dlast, gate, x, saved, initial)
