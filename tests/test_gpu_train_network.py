"""The example that runs the operators together: its gradients against autograd in 64 bits, and that it learns, with moments in 32 bits and in 8."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from cada_synth import configs
from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu


def test_gradients_of_the_whole_network():
    """bf16 activations and signals are rounded once per layer (2^-9 relative each): after four layers the gradients' 2-norm is within 3 per cent."""
    import train_network as tn
    net = tn.Network([60, 48, 48, 48, 7], act="gelu", seed=3)
    x, y = torch.randn(90, 60, device="cuda").to(torch.bfloat16), torch.randint(7, (90,), device="cuda")
    logits, kept = net.forward(x)
    loss, _, dlogits = ops.cross_entropy(logits, y, smoothing=0.1)
    net.backward(dlogits, kept)
    params = [p.double().requires_grad_() for p in net.params]
    h = x.double()
    for i, act in enumerate(net.acts):
        z = h @ params[2 * i] + params[2 * i + 1]
        z = z * torch.special.ndtr(z) if act == "gelu" else z
        h = z + h if net.residual[i] else z
    logp = torch.log_softmax(h, 1)
    want = -(0.9 * logp.gather(1, y[:, None])[:, 0] + 0.1 * logp.mean(1)).mean()
    want.backward()
    assert abs(float(loss) - want.item()) < 0.01 * abs(want.item())
    for g, p in zip(net.grads, params):
        assert float((g.double() - p.grad).norm()) <= 0.03 * float(p.grad.norm())


@pytest.mark.parametrize("bits", [32, 8])
def test_it_learns(bits):
    import train_network as tn
    cfg = configs.CFG4.scaled(name="example", layer_dims=(48, 40, 10), M=8, N_m=400, B=32, K=120, D=10)
    losses, net, opt = tn.train(cfg, 120, width=64, blocks=2, lr=2e-3, state_bits=bits)
    first, last = float(losses[:5].mean()), float(losses[-10:].mean())
    print("bits", bits, "loss", first, "->", last, "norm", float(opt.norm))
    assert torch.isfinite(losses).all() and last < 0.85 * first
    # the copies that the products read are the masters rounded
    for p, q in zip(net.masters, net.params):
        assert torch.equal(p.to(torch.bfloat16), q)


def test_8_bits_follow_32():
    """The same run with moments in 8 bits: the loss at the end within 10 per cent of that with 32."""
    import train_network as tn
    cfg = configs.CFG4.scaled(name="example", layer_dims=(48, 40, 10), M=8, N_m=400, B=32, K=120, D=10)
    ends = [float(tn.train(cfg, 120, width=64, blocks=2, lr=1e-3, state_bits=b)[0][-20:].mean()) for b in (32, 8)]
    assert abs(ends[1] - ends[0]) < 0.1 * ends[0], ends
