"""GPU: attention and its gradients where there is nothing to see, and beside
large numbers that a row or a key does not see."""
import sys

import pytest
import torch

from paper_2110_04175_amd import layer

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def announce(msg):
    sys.__stderr__.write(f"[gpu] {msg}\n")
    sys.__stderr__.flush()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,keys,heads,kv,width", [(1000, 0, 1, 1, 16), (700, 0, 6, 2, 200), (20000, 0, 4, 4, 64),
                                                        (0, 1000, 4, 1, 64), (0, 300, 2, 2, 256)])
def test_many_rows_without_keys(tokens, keys, heads, kv, width, dtype):
    """Rows of which each sees nothing, keys that nothing sees: zeros, and an lse of
    -infinity."""
    announce(f"attention of {tokens} rows and {keys} keys, {dtype}")
    q = torch.ones(2, tokens, heads, width, dtype=dtype, device="cuda")
    k = torch.ones(2, keys, kv, width, dtype=dtype, device="cuda")
    starts, none = (torch.tensor([0, at], dtype=torch.int32, device="cuda") for at in (tokens, keys))
    for ranges in (None, layer.attention_ranges(starts, tokens, none, keys)):
        out, lse = layer.attention(q, k, k, ranges)
        assert (out == 0).all() and (lse == -float("inf")).all()
        grads = layer.attention_backward(q, q, k, k, out, lse, ranges)
        for g, x in zip(grads, (q, k, k)):
            assert g.shape == x.shape and (g == 0).all()
