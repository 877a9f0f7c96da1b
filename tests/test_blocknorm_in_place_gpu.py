"""GPU: the norms around a block with results over their own inputs' rows, through
the C calls: bit for bit what they give elsewhere."""
import sys

import pytest
import torch

import paper_2110_04175_amd as rs
from paper_2110_04175_amd import layer

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
# One for each number of threads that share a row, and of chunks that a thread has.
WIDTHS = [100, 500, 1000, 1030, 3000, 4100, 7000, 12000, 20000]
N, T = 2, 37


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


def rows(t):
    return layer.Rows(t.data_ptr(), layer.TYPES[t.dtype], t.stride(0), t.stride(1))


def done(rc):
    assert rc == rs.RELAYSUM_OK, layer._lib().relaysum_layer_error().decode()


def make(seed, width, dtype):
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.empty(*shape).normal_(mean, std, generator=gen).cuda()

    x = {name: normal(N, T, width).to(dtype) for name in ("z", "gate", "residual", "dy", "dsum")}
    x |= {name: normal(N, width, std=0.1, mean=1.0) for name in ("post", "weight")}
    return x | {"scale": normal(N, mean=0.5)}


def forward(x, out):
    n, t, width = x["z"].shape
    y, saved = layer.Packed._new(n, t, width, 0, x["z"]), layer.Packed._new(n, t, width, layer.GROUP, x["z"])
    stats = torch.empty(2, n, t, device="cuda")
    done(layer._lib().relaysum_blocknorm(
        n, t, width, rows(x["z"]), rows(x["gate"]), rows(x["residual"]), x["post"].data_ptr(), width,
        x["scale"].data_ptr(), 1, x["weight"].data_ptr(), width, 1e-6, rows(out), y._c(0, "y"), stats[0].data_ptr(),
        stats[1].data_ptr(), saved._c(0, "saved"), None))
    torch.cuda.synchronize()
    return y, saved, stats


def backward(x, saved, stats, dz, dgate, ds, dsum=True):
    n, t, width = x["z"].shape
    lib = layer._lib()
    size = lib.relaysum_blocknorm_workspace(n, t, width)
    ws = torch.empty(max(size, 4), dtype=torch.uint8, device="cuda")
    dp, dw, dsc = (torch.empty(n, w, device="cuda") for w in (width, width, 1))
    grads = [layer.Rows(g.data_ptr(), layer.RELAYSUM_FLOAT, g.stride(0), 0) for g in (dp, dsc, dw)]
    done(lib.relaysum_blocknorm_backward(
        n, t, width, rows(x["dy"]), rows(x["dsum"]) if dsum else None, rows(x["z"]), rows(x["gate"]), saved._c(0, "saved"),
        stats[0].data_ptr(), stats[1].data_ptr(), x["post"].data_ptr(), width, x["scale"].data_ptr(), 1,
        x["weight"].data_ptr(), width, rows(dz), rows(dgate), rows(ds), *grads, ws.data_ptr(), size, None))
    torch.cuda.synchronize()
    return dp, dw, dsc


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_the_sum_over_an_input(width, dtype):
    announce(f"blocknorm in place width={width} {dtype}")
    x = make(1, width, dtype)
    want = torch.empty_like(x["z"])
    y, saved, stats = forward(x, want)
    for over in ("z", "gate", "residual"):
        own = x | {over: x[over].clone()}
        y2, saved2, stats2 = forward(own, own[over])
        assert torch.equal(own[over], want), over
        assert torch.equal(stats, stats2) and torch.equal(y.codes, y2.codes) and torch.equal(y.exps, y2.exps)
        assert torch.equal(saved.codes, saved2.codes) and torch.equal(saved.exps, saved2.exps)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_gradients_over_inputs(width, dtype):
    announce(f"blocknorm gradients in place width={width} {dtype}")
    x = make(2, width, dtype)
    _, saved, stats = forward(x, torch.empty_like(x["z"]))
    for dsum in (True, False):
        want = [torch.empty_like(x["z"]) for _ in range(3)]
        sums = backward(x, saved, stats, *want, dsum)
        for over in (("z", "gate", "dsum"), ("z", "gate", "dy"), ("dy", "z", "gate"), ("gate", "dy", "z")):
            if "dsum" in over and not dsum:
                continue
            own = x | {name: x[name].clone() for name in over}
            got = [own[name] for name in over]
            again = backward(own, saved, stats, *got, dsum)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), over
            assert all(torch.equal(a, b) for a, b in zip(again, sums)), over
