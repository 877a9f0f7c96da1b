"""The rule that picks a product's tile and the parts of its sum, and the
workspaces that follow from it."""
import os
import random
import shutil
import subprocess
import sys

import pytest
import torch

import paper_2110_04175_amd as rs
from paper_2110_04175_amd import layer

HERE = os.path.dirname(os.path.abspath(__file__))
LAUNCH = 0x3fffff        # workgroups of a launch
PRODUCT, INPUT, WEIGHT = 0, 1, 2


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    exe = str(tmp_path_factory.mktemp("plan") / "plan_print")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-o", exe, os.path.join(HERE, "layer_plan", "plan_print.cpp")], check=True)

    def ask(lines):
        text = "\n".join(" ".join(str(v) for v in line) for line in lines)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]

    return ask


def forward(n, tokens, width, channels):
    """The text of a product call whose arrays are no device memory: it fails,
    but not before its sizes are taken."""
    lib = layer._lib()
    far = [(5 + i) << 42 for i in range(5)]
    x, w = (layer._CPacked(a, a + (1 << 41), 0) for a in far[:2])
    y = layer.Rows(far[2], layer.RELAYSUM_BFLOAT, tokens * channels, channels)
    assert lib.relaysum_linear(n, tokens, width, channels, x, w, y, far[3], 1 << 41, None) != 0
    return lib.relaysum_layer_error().decode()


@pytest.mark.parametrize("n,tokens,width,channels", [
    (8192, 16, 64, 65536), ((1 << 20) - 1, 1, 64, 1024), (1 << 20, 70, 64, 600), ((1 << 22) - 1, 1, 64, 256)])
def test_results_that_only_the_largest_tile_fits(n, tokens, width, channels):
    """More than 2^22 small tiles, which the rule would take on their time."""
    assert "tiles" not in forward(n, tokens, width, channels)


def test_results_that_no_tile_fits():
    assert "tiles" in forward(1 << 22, 1, 64, 256)
    assert rs.RELAYSUM_MAX_WORKERS > 1 << 22


def test_every_launch_fits_where_one_can(plan):
    rng = random.Random(1)
    lines = []
    for _ in range(20000):
        n, tokens, width, channels = (int(2 ** rng.uniform(0, top)) for top in (24, 20, 15, 20))
        if n * (tokens + width) * channels < 1 << 50 and n * tokens * width < 1 << 50:
            lines.append((rng.choice([PRODUCT, INPUT, WEIGHT]), rng.choice([0, 1, 2]), n, tokens, width, channels))
    large = [(128, 128), (256, 256), (128, 256)]
    beyond = 0
    for (kind, kindtype, n, tokens, width, channels), (tile, split, blocks, workspace) in zip(lines, plan(lines)):
        m, cols = {PRODUCT: (tokens, channels), INPUT: (tokens, width), WEIGHT: (channels, width)}[kind]
        bm, bn = (256, 256) if kind == PRODUCT else large[kindtype]
        least = n * -(-m // bm) * -(-cols // bn)
        assert (blocks <= LAUNCH) == (least <= LAUNCH)
        beyond += least > LAUNCH
        assert workspace == (split * n * m * cols * 4 if split > 1 else 0)
    assert 0 < beyond < len(lines) / 2


# ---- workspaces ------------------------------------------------------------------


def test_every_call_asks_for_its_own_workspace(plan):
    lib = layer._lib()
    rng = random.Random(2)
    sizes = [(2, 3084, 3170, 5717), (1, 65536, 512, 640), (1, 1, 1, 1), (3, 0, 5, 7)]
    sizes += [tuple(int(2 ** rng.uniform(0, top)) for top in (6, 16, 13, 13)) for _ in range(300)]
    for type in (layer.RELAYSUM_FLOAT, layer.RELAYSUM_BFLOAT, layer.RELAYSUM_HALF):
        lines = [(kind, type) + size for size in sizes for kind in (PRODUCT, INPUT, WEIGHT)]
        want = [p[3] for p in plan(lines)]
        got = [lib.relaysum_linear_workspace_of(kind, *size, type) for size in sizes for kind in (PRODUCT, INPUT, WEIGHT)]
        assert got == want
        most = [lib.relaysum_linear_workspace(*size, type) for size in sizes]
        assert most == [max(got[i:i + 3]) for i in range(0, len(got), 3)]


def test_workspace_queries_refuse():
    lib = layer._lib()
    for args in ((3, 1, 1, 64, 64, 0), (-1, 1, 1, 64, 64, 0), (0, 0, 1, 64, 64, 0), (1, 1, -1, 64, 64, 0),
                 (2, 1, 1, 32769, 64, 0), (0, 1, 1, 64, 0, 0), (0, 1, 1, 64, 64, 3)):
        assert lib.relaysum_linear_workspace_of(*args) == -1
        assert lib.relaysum_layer_error()
    assert lib.relaysum_linear_workspace_of(0, 1, 1, 64, 64, 0) >= 0
    assert lib.relaysum_layer_error() == b""


@pytest.mark.gpu
def test_calls_allocate_what_they_need():
    """Sizes at which only one of the three calls makes its sum in parts: the
    others take their results' memory and no more (allocations are rounded up
    to 2 MiB at most)."""
    sys.__stderr__.write("[gpu] memory of the products' calls\n")
    sys.__stderr__.flush()
    n, tokens, width, channels = 2, 3084, 3170, 5717
    code = layer.RELAYSUM_BFLOAT
    need = [layer._lib().relaysum_linear_workspace_of(p, n, tokens, width, channels, code) for p in (PRODUCT, INPUT, WEIGHT)]
    assert need[PRODUCT] == 0 and need[WEIGHT] == 0 and need[INPUT] > 100 << 20
    x = layer.pack(torch.zeros(n, tokens, width, device="cuda"))
    w = layer.pack(torch.zeros(n, channels, width, device="cuda"))
    dy = torch.zeros(n, tokens, channels, device="cuda", dtype=torch.bfloat16)
    dw = torch.zeros(n, channels, width, device="cuda")
    for call, result in ((lambda: layer.linear(x, w), dy.numel() * 2), (lambda: layer.linear_backward_weight(dy, x, dw), 0),
                         (lambda: layer.linear_backward_input(dy, w), n * tokens * width * 2 + need[INPUT])):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        call()
        torch.cuda.synchronize()
        assert torch.cuda.max_memory_allocated() - before <= result + (4 << 20)
