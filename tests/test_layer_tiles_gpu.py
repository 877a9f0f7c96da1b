"""GPU: every tile of the products and their gradients, with and without a sum
in parts, against products in 64 bits; and the scaling of the integer product
over all exponents in each of its tiles.

Bounds are those of test_layer_gpu.py: the product is exact, a gradient is off
by its additions' roundings."""
import os
import shutil
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2110_04175_amd import layer
from test_layer_gpu import ROUND, TINY, TYPES, ULP, in_64, in_model, random_codes, untouched

HERE = os.path.dirname(os.path.abspath(__file__))

# n, tokens, width, channels.  The tiles of 16 x 128, 64 x 128 and 256 x 256, each whole and in parts.
PRODUCTS = [(3, 33, 517, 201), (2, 9, 3001, 133), (3, 1000, 1001, 777), (30, 620, 519, 37), (36, 241, 2445, 25),
            (43, 519, 70, 130), (7, 1030, 300, 770), (3, 4199, 7604, 132), (1, 1171, 6475, 6396)]
# By dY's type, the small tile and the large one, each whole and in parts.
SMALL = [(3, 70, 100, 33), (2, 37, 130, 901), (2, 1601, 130, 37)]
GRADIENTS = {torch.float32: SMALL + [(12, 605, 397, 65), (23, 8, 129, 285), (3, 65, 135, 4733), (23, 302, 136, 3)],
             torch.bfloat16: SMALL + [(35, 717, 140, 4), (14, 417, 143, 1958), (7, 195, 3658, 2431), (10, 30, 5860, 65),
                                      (2, 6006, 132, 1353)],
             torch.float16: SMALL + [(24, 67, 1507, 21), (36, 69, 151, 438), (27, 8, 137, 587), (18, 776, 135, 145)]}
# Of one step: tokens and channels for each tile.
SCALED = {2: (1, 37, 128, 201), 1: (3, 5582, 128, 1), 0: (43, 519, 128, 130)}


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


def test_sizes_reach_every_tile(tmp_path):
    """On the CPU: what the rule picks for the sizes of this file."""
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    exe = str(tmp_path / "plan_print")
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", exe, os.path.join(HERE, "layer_plan", "plan_print.cpp")], check=True)
    lines = [(0, 0) + size for size in PRODUCTS + list(SCALED.values())]
    lines += [(kind, layer.TYPES[dtype]) + size for kind in (1, 2) for dtype, sizes in GRADIENTS.items() for size in sizes]
    text = "\n".join(" ".join(str(v) for v in line) for line in lines)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    plans = [tuple(int(v) for v in line.split()) for line in out]
    for tile, got in zip(SCALED, plans[len(PRODUCTS):]):
        assert got[:2] == (tile, 1)
    kinds = [(kind, type if kind else 0) for kind, type, *_ in lines]
    reached = {(kind, type, tile, split > 1) for (kind, type), (tile, split, *_) in zip(kinds, plans)}
    wanted = {(0, 0, tile, parts) for tile in range(3) for parts in (False, True)}
    wanted |= {(kind, type, tile, parts) for kind in (1, 2) for type in range(3) for tile in range(2) for parts in (False, True)}
    assert reached == wanted, wanted - reached


@pytest.mark.gpu
@pytest.mark.parametrize("n,tokens,width,channels", PRODUCTS)
def test_product(n, tokens, width, channels):
    announce(f"product {n} {tokens} {width} {channels}")
    x, w = random_codes(1, n, tokens, width), random_codes(2, n, channels, width)
    want = torch.matmul(in_64(x), in_64(w).transpose(1, 2).contiguous())
    for dtype in TYPES:
        assert torch.equal(layer.linear(x, w, dtype), want.float().to(dtype)), dtype


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,size", [(dtype, size) for dtype, sizes in GRADIENTS.items() for size in sizes])
def test_gradients(dtype, size):
    n, tokens, width, channels = size
    announce(f"gradients {size} {dtype}")
    w = random_codes(2, n, channels, width)
    g = torch.Generator(device="cuda").manual_seed(3)
    dy = (torch.randn(n, tokens, channels, generator=g, device="cuda") * 1e-2).to(dtype)
    d64, w64 = dy.double(), in_64(w)
    want, size = torch.matmul(d64, w64), torch.matmul(d64.abs(), w64.abs())
    bound = 2 * (channels + 8) * ULP * size + 1.01 * ROUND[dtype] * want.abs() + TINY[dtype]
    assert bool(((layer.linear_backward_input(dy, w).double() - want).abs() <= bound).all())
    turned = d64.transpose(1, 2).contiguous()
    for group in (0, 128):
        x = random_codes(4, n, tokens, width, group)
        dw, around = in_model(torch.zeros(n, channels, width, device="cuda"))
        layer.linear_backward_weight(dy, x, dw)
        x64 = in_64(x)
        want, size = torch.matmul(turned, x64), torch.matmul(turned.abs(), x64.abs())
        assert bool(((dw.double() - want).abs() <= 2 * (tokens + 8) * ULP * size).all())
        assert untouched(dw, around)


# Up to 98 a code sum times 2^ex is a normal number; tokens beyond take their wave another way.
TOKENS = {"up to 98": [-126, -125, -60, 0, 60, 97, 98, -128], "beyond": [-126, -60, 0, 97, 98, 99, 110, 122, -128]}


@pytest.mark.gpu
@pytest.mark.parametrize("tile", sorted(SCALED))
@pytest.mark.parametrize("which", TOKENS)
def test_product_over_all_exponents(tile, which):
    """Codes over their whole range; results from zero past the smallest
    numbers to infinities, and NaN for tokens and channels that are NaN."""
    n, tokens, width, channels = SCALED[tile]
    announce(f"product's scales, tile {tile}, tokens' exponents {which}")
    g = np.random.default_rng(tile)
    qx = g.integers(-127, 128, (n, tokens, width)).astype(np.int8)
    qw = g.integers(-127, 128, (n, channels, width)).astype(np.int8)
    qx[:, -1] = 127
    qw[:, -1] = -127
    ex = g.choice(TOKENS[which], (n, tokens, 1)).astype(np.int8)
    ew = g.choice([-126, -125, -90, -40, 0, 3, 40, 90, 99, 122, -128], (n, channels, 1)).astype(np.int8)
    if channels == 1:
        ew[:, 0, 0] = [-100, 0, 40]       # one channel of each worker: not all of them NaN
    x = layer.Packed(torch.from_numpy(qx).cuda(), torch.from_numpy(ex).cuda(), width)
    w = layer.Packed(torch.from_numpy(qw).cuda(), torch.from_numpy(ew).cuda(), width)
    sums = np.matmul(qx.astype(np.float64), qw.astype(np.float64).transpose(0, 2, 1))
    e = ex.astype(np.int64) + ew.astype(np.int64).transpose(0, 2, 1)
    nan = (ex == -128) | (ew == -128).transpose(0, 2, 1)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(np.where(nan, np.nan, np.ldexp(sums, np.where(nan, 0, e))).astype(np.float32))
    assert bool(torch.isnan(want).any()) and bool((want == 0).any()) and bool(torch.isfinite(want).any())
    assert bool(((want != 0) & (want.abs() < 2.0 ** -126)).any()) and bool(torch.isinf(want).any())
    for dtype in TYPES:
        got = layer.linear(x, w, dtype).cpu()
        torch.testing.assert_close(got, want.to(dtype), rtol=0, atol=0, equal_nan=True)
