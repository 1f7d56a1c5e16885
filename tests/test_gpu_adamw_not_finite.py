"""Infinities in the AdamW step: 8-bit codes do not turn one into something finite later, and the fill behind a tensor's moments keeps its zeros whatever the gradients are."""
import math

import pytest
import torch

from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [math.inf, -math.inf, 3e38], ids=str)
def test_a_block_with_an_infinity_is_not_a_number(value):
    """3e38: finite, but its square is not in float32, so the second moment is infinite and the first is not."""
    params, grads = [torch.ones(1000, device="cuda")], [torch.full((1000,), 0.1, device="cuda")]
    grads[0][300] = value
    grads[0][400:410] = 0.0
    opt = ops.AdamW(params, grads, state_bits=8)
    opt.step()
    m, v = opt.moments()
    assert torch.isnan(v[256:512]).all() and (math.isfinite(value) or torch.isnan(m[256:512]).all())
    for x in (m, v):
        assert torch.isfinite(x[:256]).all() and torch.isfinite(x[512:]).all()
    grads[0].fill_(0.1)
    opt.step()          # the block does not recover, the others go on
    assert torch.isnan(params[0][256:512]).all() and torch.isfinite(params[0][:256]).all() and torch.isfinite(params[0][512:]).all()
    assert torch.isnan(opt.moments()[1][256:512]).all()


@pytest.mark.parametrize("types", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)], ids=str)
@pytest.mark.parametrize("clip", [0.0, 1.0])
def test_the_fill_keeps_its_zeros(types, clip):
    sizes = [1, 3, 8, 250, 255, 257, 2049, 5000]
    for bad, scale in ((math.nan, 1.0), (math.inf, 1.0), (0.1, math.inf), (0.1, math.nan)):
        params, grads = [torch.ones(n, device="cuda", dtype=types[0]) for n in sizes], [torch.full((n,), 0.1, device="cuda", dtype=types[1]) for n in sizes]
        for g in grads:
            g[-1] = bad
        opt = ops.AdamW(params, grads, max_norm=clip)
        opt.step(grad_scale=torch.tensor([scale], device="cuda"))
        for x in opt.moments():
            for n, at in zip(sizes, opt.offsets):
                assert not x[at + n:at + -(-n // 256) * 256].any()
                assert not torch.isfinite(x[at + n - 1])
