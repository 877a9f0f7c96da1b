"""GPU: the sum of a block norm in 16 bits is the float sum of the same rows, rounded."""
import sys

import pytest
import torch

from paper_2110_04175_amd import layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_the_sum_is_the_float_sum_rounded(dtype, gated):
    """Bit for bit, of two million entries: both norms' factors follow."""
    sys.__stderr__.write(f"[gpu] blocknorm's sum rounded {dtype} {gated}\n")
    sys.__stderr__.flush()
    n, t, w = 4, 512, 1024
    gen = torch.Generator().manual_seed(5)
    z, gate, residual = (torch.empty(n, t, w).normal_(generator=gen).to(dtype).cuda() for _ in range(3))
    post, weight = (torch.empty(n, w).normal_(1.0, 0.1, generator=gen).cuda() for _ in range(2))
    scale = torch.empty(n).normal_(0.5, 0.1, generator=gen).cuda()
    gate = gate if gated else None
    s, y, post_rstd, rstd, _ = layer.blocknorm(z, gate, residual, post, scale, weight)
    wide = [None if v is None else v.float() for v in (z, gate, residual)]
    s32, _, post32, _, _ = layer.blocknorm(*wide, post, scale, weight)
    assert torch.equal(s, s32.to(dtype)), int((s != s32.to(dtype)).sum())
    assert torch.equal(post_rstd, post32)
    _, y32, rstd32, _ = layer.rmsnorm(s.float(), None, weight)
    assert torch.equal(rstd, rstd32) and torch.equal(y.exps, y32.exps) and torch.equal(y.codes, y32.codes)
