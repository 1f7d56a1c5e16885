"""The embedding's, layer norm's and the last layer's loss on streams: one of another device than the operands' is refused; calls that overlap on two streams; what a call is not asked for is not read."""
import types

import pytest
import torch

from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu


def calls():
    x, v, t = torch.randn(8, 8, device="cuda"), torch.ones(8, device="cuda"), torch.zeros(8, dtype=torch.int64, device="cuda")
    return [lambda s: ops.layer_norm_forward(x, stream=s), lambda s: ops.layer_norm_backward(x, x, v, v, stream=s), lambda s: ops.embedding_forward(t, x, stream=s),
            lambda s: ops.embedding_backward(x, t, 8, stream=s), lambda s: ops.linear_cross_entropy(x, x, t, stream=s)]


@pytest.mark.parametrize("which", range(5))
def test_a_stream_of_another_device(which):
    call = calls()[which]
    with pytest.raises(ValueError, match="stream must be one of cuda:0's"):
        call(types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0))
    call(torch.cuda.Stream())
    torch.cuda.synchronize()


def test_two_at_once():
    """The same calls on two streams, each with workspaces of its own, while the other's are under way."""
    gen = torch.Generator(device="cuda"); gen.manual_seed(1)
    x, w = torch.randn(2000, 256, generator=gen, device="cuda").to(torch.bfloat16), torch.randn(256, 9000, generator=gen, device="cuda").to(torch.bfloat16)
    labels, tokens = torch.randint(9000, (2000,), generator=gen, device="cuda"), torch.randint(500, (2000,), generator=gen, device="cuda")
    mean, rstd = ops.layer_norm_forward(x, keep_stats=True)[1:]

    def all_of(s=None):
        return (*ops.linear_cross_entropy(x, w, labels, smoothing=0.1, stream=s)[:4], ops.embedding_backward(x, tokens, 500, stream=s), *ops.layer_norm_backward(x, x, mean, rstd, stream=s))

    want = all_of()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[all_of(s) for s in streams] for _ in range(4)]
    torch.cuda.synchronize()
    for pair in got:
        for out in pair:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_a_workspace_of_ones_own():
    """Handed in, and with whatever in it."""
    x, w, labels = torch.randn(300, 64, device="cuda"), torch.randn(64, 700, device="cuda"), torch.randint(700, (300,), device="cuda")
    mean, rstd = ops.layer_norm_forward(x, keep_stats=True)[1:]
    for call in (lambda **k: ops.linear_cross_entropy(x, w, labels, **k)[:4], lambda **k: ops.layer_norm_backward(x, x, mean, rstd, **k), lambda **k: (ops.embedding_backward(torch.cat([x, x]), torch.cat([labels, labels]), 700, **k),)):
        want = call()
        for fill in (0, 255):
            ws = torch.full((1 << 24,), fill, dtype=torch.uint8, device="cuda")
            assert all(torch.equal(a, b) for a, b in zip(call(workspace=ws), want))
            assert all(torch.equal(a, b) for a, b in zip(call(workspace=ws), want))
