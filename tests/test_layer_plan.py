"""CPU: the rule that picks a product's tile and the parts of its sum."""
import os
import random
import shutil
import subprocess

import pytest

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
