"""Outputs of the layer calls may lie between other arrays' rows, but share no
entry with them."""
import sys

import numpy as np
import pytest
import torch

import paper_2110_04175_amd as rs
from paper_2110_04175_amd import layer

BASE = 1 << 34


def norm_backward(n, width, weight, weight_stride, grad, grad_stride):
    lib = layer._lib()
    far = [(5 + i) << 36 for i in range(4)]
    dy, ds = layer.Rows(far[0], 0, width, width), layer.Rows(far[1], 0, width, width)
    saved = layer._CPacked(far[2], far[2] + (1 << 34), 128)
    rc = lib.relaysum_rmsnorm_backward(n, 1, width, dy, None, saved, far[3], weight, weight_stride, ds,
                                       layer.Rows(grad, 0, grad_stride, 0), None, 0, None)
    return rc, lib.relaysum_layer_error().decode()


# The addresses are not device memory, so every call fails in the end: without
# a GPU when it asks for one, else when it looks the addresses up.  Arrays that
# share entries are refused before that.

@pytest.mark.parametrize("at,stride,shares", [
    (100, 200, False),      # halves of one tensor [n][2 * 100]
    (-100, 200, False),
    (99, 200, True), (-99, 200, True), (101, 200, True), (0, 200, True),
    (100, 201, True),       # another stride runs into the rows
    (40, 400, True), (100, 400, False), (300, 400, False), (301, 400, True), (-60, 400, True),
    (100, 600, False),      # every third gap
    (500, 200, False), (580, 200, True), (700, 200, False),
])
def test_weight_gradients_between_the_rows_of_weights(at, stride, shares):
    """5 rows of 100 weights, 200 apart (400 where the gradients' are)."""
    weight_stride = 400 if stride == 400 else 200
    rc, text = norm_backward(5, 100, BASE, weight_stride, BASE + 4 * at, stride)
    weights = {i * weight_stride + k for i in range(5) for k in range(100)}
    grads = {at + i * stride + k for i in range(5) for k in range(100)}
    if shares:
        assert weights & grads
        assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "share memory" in text
    else:
        assert not weights & grads
        assert rc != 0 and "share memory" not in text


@pytest.mark.parametrize("at,shares", [(400, False), (608, False), (2400, False), (384, True), (624, True), (1008, True)])
def test_codes_between_rows(at, shares):
    """384 bytes of codes beside 3 rows of 100 floats, 250 apart."""
    lib = layer._lib()
    rc = lib.relaysum_pack(1, 3, 100, layer.Rows(BASE, 0, 0, 250), layer._CPacked(BASE + at, BASE << 2, 0), None)
    text = lib.relaysum_layer_error().decode()
    assert rc != 0 and ("share memory" in text) == shares


@pytest.mark.parametrize("seed", range(40))
def test_random_layouts(seed):
    """Sets of entries written out: what shares one is always refused, and two
    parts of one tensor [workers][rows][wide] or [rows][workers][wide] never."""
    rng = np.random.default_rng(seed)
    for _ in range(20):
        n, width, rows = (int(v) for v in rng.integers(1, 6, 3))
        wide = 2 * width + int(rng.integers(0, 3))
        a = int(rng.integers(0, wide - 2 * width + 1))
        b = a + width + int(rng.integers(0, wide - 2 * width - a + 1))
        inside = rng.random() < 0.5
        ws, rs_ = (rows * wide, wide) if inside else (wide, n * wide)
        if rng.random() < 0.3:
            b = int(rng.integers(-width, 2 * width))
        lib = layer._lib()
        x, y = layer.Rows(BASE + 4 * a, 0, ws, rs_), layer.Rows(BASE + 4 * b, 0, ws, rs_)
        far = [(5 + i) << 36 for i in range(6)]
        # h and residual in, sum out; sum may be h itself, so residual is what is tried.
        rc = lib.relaysum_rmsnorm(n, rows, width, layer.Rows(far[0], 0, rows * width, width), x, far[1], width,
                                  1e-6, y, layer._CPacked(far[2], far[3], 0), far[4], None, None)
        text = lib.relaysum_layer_error().decode()

        def entries(start):
            return {start + i * ws + t * rs_ + k for i in range(n) for t in range(rows) for k in range(width)}

        if a != b and entries(a) & entries(b):
            assert rc == rs.RELAYSUM_ERR_INVALID_ARG and "share memory" in text
        else:
            assert rc != 0 and "share memory" not in text, (n, rows, width, wide, a, b, inside)


@pytest.mark.gpu
def test_models_and_gradients_in_one_tensor():
    """x and g as halves of one tensor [n][2d]: the same bits as apart, and
    the models stay."""
    sys.__stderr__.write("[gpu] models and gradients in one tensor\n")
    sys.__stderr__.flush()
    n, t, k, c = 3, 40, 70, 50
    d = k + c * k + 1
    gen = torch.Generator(device="cuda").manual_seed(1)
    both = torch.randn(n, 2 * d, generator=gen, device="cuda")
    kept = both.clone()
    apart = torch.zeros(n, d, device="cuda")
    x = both[:, :d]
    h = torch.randn(n, t, k, generator=gen, device="cuda")
    dy = torch.randn(n, t, c, generator=gen, device="cuda")
    w = layer.pack(x[:, k:k + c * k].unflatten(1, (c, k)))
    s, y, rstd, saved = layer.rmsnorm(h, None, x[:, :k])
    dn = layer.linear_backward_input(dy, w)
    for g in (apart, both[:, d:]):
        layer.linear_backward_weight(dy, y, g[:, k:k + c * k].unflatten(1, (c, k)))
        layer.rmsnorm_backward(dn, None, saved, rstd, x[:, :k], g[:, :k])
    assert torch.equal(both[:, d:2 * d - 1], apart[:, :d - 1])
    assert torch.equal(both[:, :d], kept[:, :d]) and torch.equal(both[:, -1], kept[:, -1])
    with pytest.raises(rs.RelaySumError):
        layer.rmsnorm_backward(dn, None, saved, rstd, x[:, :k], both[:, k - 1:2 * k - 1])
