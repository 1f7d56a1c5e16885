"""Where the values of a plan's moments may be written."""
import pytest
import torch

from paper_2012_15469_amd import ops
from paper_2012_15469_amd.binding import _lib, cada_last_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
def test_values_that_share_memory_are_refused(bits):
    params, grads = [torch.ones(5000, device="cuda")], [torch.ones(5000, device="cuda")]
    opt = ops.AdamW(params, grads, state_bits=bits)
    opt.step()
    a, b = torch.zeros(2 * 5120, device="cuda"), torch.zeros(5120, device="cuda")
    held = [x for s in (opt.m, opt.v) for x in (s if bits == 8 else (s,))] + [opt.workspace]
    before = [x.clone() for x in held]
    for m, v in [(a, a), (a, a[5119:])] + [(x, None) for x in held] + [(None, x) for x in held]:
        assert _lib.cada_adamw_moments(opt.plan, None if m is None else m.data_ptr(), None if v is None else v.data_ptr()) == -1 and "share memory" in cada_last_error()
    assert all(torch.equal(x, y) for x, y in zip(held, before))
    assert _lib.cada_adamw_moments(opt.plan, a.data_ptr(), a[5120:].data_ptr()) == 0 and _lib.cada_adamw_moments(opt.plan, b.data_ptr(), None) == 0
    m, v = opt.moments()
    assert torch.equal(a[:5120], m) and torch.equal(a[5120:], v) and torch.equal(b, m)
