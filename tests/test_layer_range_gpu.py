"""GPU: the layer operators at both ends of the floats' range, against their
plain 64-bit implementations (oracle/layer.py).

Tolerances are those of test_layer_gpu.py.  Where a result or an entry lies
below the smallest normal number its own type's smallest step is added."""
import sys

import numpy as np
import pytest
import torch

from oracle import layer as plain
from paper_2110_04175_amd import layer
from test_layer_gpu import ROUND, TINY, ULP, held, in_model, normal, same_packed

pytestmark = pytest.mark.gpu

LARGEST = 3.4028234663852886e38


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


def host(t):
    return t.double().cpu().numpy()


# ---- the norm: mean squares past binary32's range on either side -----------------

# Factors of a row of normal entries, and eps: the sum of squares overflows
# while its mean does not (1e18), both overflow, squares lose bits below the
# smallest normal number or vanish; in the last two eps is larger than they are.
NORM_ROWS = [(1e18, 1e-6), (1e19, 1e-6), (3e37, 0.0), (1e-21, 0.0), (1e-25, 0.0), (1e-37, 0.0), (1e-15, 0.0),
             (1e-25, 1e-42), (1e-30, 1e-38)]


@pytest.mark.parametrize("width", [1, 100, 1001, 4100, 32768])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_of_large_and_small_rows(width, dtype):
    """A row of ordinary size beside each, so that rows share a wave."""
    for factor, eps in NORM_ROWS:
        announce(f"norm width={width} {dtype} factor={factor} eps={eps}")
        h = normal(1, 2, 3, width)
        h[1] *= factor
        h[0, 1] *= factor
        # 5 * 3e37 and a residual of a tenth of that stay below the largest number.
        h = h.clamp(-5 * factor, 5 * factor).to(dtype) if factor > 5 else h.to(dtype)
        w = 1 + 0.1 * normal(3, 2, width)
        r = normal(2, 2, 3, width, std=0.1)
        r[1] *= factor
        r[0, 1] *= factor
        for residual in (None, r.to(dtype)):
            s, y, rstd, saved = layer.rmsnorm(h, residual, w, eps)
            sh = host(s)
            assert np.isfinite(sh).all()
            assert same_packed(saved, plain.pack(sh, 128))
            want, want_rstd = plain.rmsnorm(sh, host(w), float(np.float32(eps)))
            rel = (min(width, 42) + 8) * ULP
            with np.errstate(over="ignore"):
                np.testing.assert_allclose(host(rstd), want_rstd.astype(np.float32).astype(np.float64),
                                           rtol=rel + 2 * ULP, atol=2 * TINY[torch.float32])
            e = y.exps.cpu().numpy().astype(np.int64)
            off = np.abs(plain.values(y.codes.cpu().numpy(), y.exps.cpu().numpy(), width) - want)
            assert (off <= 0.5 * 2.0 ** e + (rel + 4 * ULP) * np.abs(want)).all()
            top = np.max(np.abs(want), axis=2, keepdims=True)
            assert (top * (1 + 2 * rel + 4 * ULP) > 127 * 2.0 ** (e - 1)).all()


def test_norm_gradient_of_a_large_row():
    """A row whose squares sum past the range takes its part in the weight's
    gradient."""
    announce("norm gradient of a large row")
    n, t, k = 1, 3, 1000
    h = normal(1, n, t, k)
    h[0, 1] *= 1e18
    w, dw = torch.ones(n, k, device="cuda"), torch.zeros(n, k, device="cuda")
    s, y, rstd, saved = layer.rmsnorm(h, None, w, 1e-6)
    dy = normal(2, n, t, k)
    ds = layer.rmsnorm_backward(dy, None, saved, rstd, w, dw)
    want, want_dw = plain.rmsnorm_backward(host(dy), None, held(saved), host(rstd), host(w))
    xh = np.abs(held(saved)) * host(rstd)[:, :, None]
    assert (np.abs(xh[0, 1]).max() > 1)
    u = np.abs(host(dy))
    size = host(rstd)[:, :, None] * (u + xh * np.mean(u * xh, axis=2, keepdims=True))
    assert (np.abs(host(ds) - want) <= 70 * ULP * size + TINY[torch.float32]).all()
    assert (np.abs(host(dw) - want_dw) <= (t + 8) * ULP * np.sum(u * xh, axis=1)).all()


# ---- the products' gradients: dY at both ends of its type's range -----------------


def check_gradients(dy, w, x):
    """dX and dW of the packed w and x, within the bound of their additions,
    and of what floats lose below 2^-133."""
    a, lost = host(dy), 2.0 ** -134 if dy.dtype == torch.float32 else 0.0
    channels, tokens = dy.shape[2], dy.shape[1]
    dx = layer.linear_backward_input(dy, w)
    b = held(w)
    want, size = np.matmul(a, b), np.matmul(np.abs(a), np.abs(b))
    bound = 2 * (channels + 8) * ULP * size + 1.01 * ROUND[dy.dtype] * np.abs(want) + TINY[dy.dtype]
    bound = bound + lost * np.sum(np.abs(b), axis=1, keepdims=True)
    assert (np.abs(host(dx) - want) <= bound).all()
    dw, _ = in_model(torch.zeros(dy.shape[0], channels, x.width, device="cuda"))
    layer.linear_backward_weight(dy, x, dw)
    a, b = a.transpose(0, 2, 1), held(x)
    want, size = np.matmul(a, b), np.matmul(np.abs(a), np.abs(b))
    bound = 2 * (tokens + 8) * ULP * size + TINY[torch.float32] + lost * np.sum(np.abs(b), axis=1, keepdims=True)
    assert (np.abs(host(dw) - want) <= bound).all()


def uniform(seed, *shape):
    g = np.random.default_rng(seed).uniform(-1, 1, shape)
    return torch.from_numpy(g.astype(np.float32)).cuda()


@pytest.mark.parametrize("factor", [1e-34, 1e-37, 1e-39, 1e-41])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_small_entries(dtype, factor):
    """Entries below the smallest normal number among them; the products of
    every multiple of 2^-133 with the rows' values are whole multiples of the
    smallest float."""
    announce(f"gradients of entries of {factor} {dtype}")
    n, t, k, c = 2, 70, 130, 90
    w, x = layer.pack(normal(1, n, c, k)), layer.pack(normal(2, n, t, k), 128)
    dy = (uniform(3, n, t, c).double() * factor).to(dtype)
    # 1e-41 lies below half of the smallest bfloat16: all of it rounds to 0.
    assert bool((dy != 0).any()) == (dtype == torch.float32 or factor > 1e-40)
    check_gradients(dy, w, x)


def test_gradients_of_the_smallest_halves():
    announce("gradients of the smallest binary16")
    n, t, k, c = 2, 70, 130, 90
    w, x = layer.pack(normal(1, n, c, k)), layer.pack(normal(2, n, t, k), 128)
    check_gradients((uniform(3, n, t, c) * 1e-6).half(), w, x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gradients_of_the_largest_entries(dtype):
    """Finite entries up to the type's largest number: small values take them
    back into the range, and zeros (a channel, a token, single entries) give
    zeros of them."""
    announce(f"gradients of the largest {dtype}")
    n, t, k, c = 2, 70, 130, 90
    top = torch.finfo(dtype).max
    wv, xv = normal(1, n, c, k, std=2.0 ** -20), normal(2, n, t, k, std=2.0 ** -20)
    wv[:, 5] = 0
    xv[:, 7] = 0
    wv[:, :, 100:] = 0
    xv[:, :, 100:] = 0
    dy = (uniform(3, n, t, c).double() * top).to(dtype)
    dy[0, 2:9, 1:40] = top
    dy[1, :, 5] = -top
    dy[:, 7] = top
    assert bool(torch.isfinite(dy).all())
    for group in (0, 128):
        check_gradients(dy, layer.pack(wv), layer.pack(xv, group))
    dx = layer.linear_backward_input(dy, layer.pack(wv))
    assert bool((dx[:, :, 100:] == 0).all())


def test_what_is_no_number_in_a_floats_last_bits():
    """NaN whose payload lies in the lower half of its bits."""
    announce("NaN in the last bits")
    dy = torch.ones(1, 40, 24, device="cuda")
    dy.view(torch.int32)[0, 3, 4] = 0x7f800001
    dx = layer.linear_backward_input(dy, layer.pack(torch.ones(1, 24, 40, device="cuda")))
    assert bool(torch.isnan(dx[0, 3]).all()) and bool((dx[0, 4:] == 24).all())
