"""GPU: how far every gradient of a block's training step has the right size."""
import pytest

import test_layer_block_gpu as block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", [1, 2])
def test_gradients_have_the_right_size(seed):
    """The part of a gradient along the one in 64 bits without 8-bit rows, over that
    one's size: 1 but for what errors add up to along it.  They are some 3% of a
    gradient's size, in all directions: over 96 entries or more 0.3% along one that
    they know nothing of, and 3% at most along any.  A term that is a twentieth too
    large, or a factor, would show."""
    block.announce(f"sizes of a block's gradients {seed}")
    data = block.make(seed)
    got, want = block.step(*data), block.plain_step(*data)
    for a, b, name in zip(got, want, ("out", "last", "sum", "x", "h", "initial")):
        a = a.double().cpu()
        parts = [(name, a, b)] if name != "x" else \
            [(part, u, v) for (part, u), v in zip(block.views(a)[0].items(), block.views(b)[0].values()) if u[0].numel() >= 96]
        for what, u, v in parts:
            for i in range(block.N):
                along = float((u[i] * v[i]).sum() / v[i].square().sum())
                block.announce(f"{what} {i}: {along:.4f}")
                assert abs(along - 1) < 0.03, (what, i, along)
