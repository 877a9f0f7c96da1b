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
# while their mean does not (1e18), both overflow, squares are below every
# normal number, or below every number; with the last of an eps that is larger.
NORM_ROWS = [(1e18, 1e-6), (1e19, 1e-6), (3e37, 0.0), (1e-21, 0.0), (1e-25, 0.0), (1e-37, 0.0), (1e-25, 1e-42),
             (1e-15, 0.0), (1e-30, 1e-38)]


@pytest.mark.parametrize("width", [1, 100, 1001, 4100, 32768])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_of_large_and_small_rows(width, dtype):
    """A row of ordinary size beside each, so that rows share a wave."""
    for factor, eps in NORM_ROWS:
        announce(f"norm width={width} {dtype} factor={factor} eps={eps}")
        h = normal(1, 2, 3, width)
        h[1] *= factor
        h[0, 1] *= factor
        # At most 2.7 sigma below the largest number's 9, so none overflows.
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
