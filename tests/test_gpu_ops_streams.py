"""A stream of another device than the operands' is refused: work would go to that device."""
import types

import pytest
import torch

from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", [
    lambda x, s: ops.linear_forward(x, x, stream=s), lambda x, s: ops.linear_backward(x, x, x, stream=s), lambda x, s: ops.cross_entropy(x, torch.zeros(8, dtype=torch.int64, device="cuda"), stream=s),
    lambda x, s: ops.AdamW([x], [x.clone()], stream=s)])
def test_a_stream_of_another_device(call):
    x = torch.zeros(8, 8, device="cuda")
    with pytest.raises(ValueError, match="stream must be one of cuda:0's"):
        call(x, types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0))
    call(x, torch.cuda.Stream())
    torch.cuda.synchronize()
