"""The example that runs the embedding, layer norm, layers and the loss without logits together: its gradients against autograd in 64 bits, its steps in a captured graph, a single row's answer."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu


def definition(net, params, tokens, labels, smoothing, ignore):
    def gelu(z):
        return z * torch.special.ndtr(z)

    def norm(x, g, s):
        c = x - x.mean(1, keepdim=True)
        return c / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-5) * g + s

    x = gelu((params[0][tokens.reshape(-1)] * net.scale).view(tokens.shape[0], -1) @ params[1] + params[2])
    for b in range(net.blocks):
        g, s, w, bias = params[3 + 4 * b:7 + 4 * b]
        x = gelu(norm(x, g, s) @ w + bias) + x
    logp = torch.log_softmax(norm(x, params[-4], params[-3]) @ params[-2] + params[-1], 1)
    used = labels != ignore
    rows = -((1 - smoothing) * logp.gather(1, labels.clamp(min=0)[:, None])[:, 0] + smoothing * logp.mean(1))
    return (rows * used).sum() / used.sum()


@pytest.mark.parametrize("vocab,width,rows", [(97, 40, 70), (1003, 72, 300)])
def test_gradients_of_the_whole_network(vocab, width, rows):
    """bf16 activations and signals are rounded once per operator (2^-8 relative at most each, in random directions): after eight of them the gradients' 2-norm is within 3 per cent."""
    import train_tokens as tt
    net = tt.TokenNetwork(vocab, width, seed=5)
    for p in net.params[-4::-4]:
        p += 0.1 * torch.randn_like(p)
    tokens, labels = torch.randint(vocab, (rows, 2), device="cuda"), torch.randint(vocab, (rows,), device="cuda")
    labels[::7] = -100
    loss = net.loss(tokens, labels, smoothing=0.1)
    params = [p.double().requires_grad_() for p in net.params]
    want = definition(net, params, tokens, labels, 0.1, -100)
    want.backward()
    assert abs(float(loss) - want.item()) < 0.01 * abs(want.item())
    for i, (g, p) in enumerate(zip(net.grads, params)):
        off = float((g.double() - p.grad).norm() / p.grad.norm())
        assert off <= 0.03, (i, off)


def test_it_runs_with_moments_of_either_kind():
    import train_tokens as tt
    for bits in (32, 8):
        losses, net, opt = tt.train(6, vocab=500, width=64, rows=256, state_bits=bits)
        assert bool(torch.isfinite(losses).all()) and all(torch.equal(p.to(torch.bfloat16), q) for p, q in zip(net.masters, net.params))
    one = net.answer(torch.tensor([[3, 4]], device="cuda"))
    assert one.shape == (1,) and 0 <= int(one) < 500


def test_steps_in_a_captured_graph():
    """Forward, backward and the optimiser's step in one graph, against the same steps made one by one."""
    import train_tokens as tt
    rows, vocab = 200, 700
    data = [(torch.randint(vocab, (rows, 2), device="cuda"), torch.randint(vocab, (rows,), device="cuda")) for _ in range(4)]
    stream = torch.cuda.Stream()
    results = []
    for captured in (False, True):
        with torch.cuda.stream(stream):
            net = tt.TokenNetwork(vocab, 64, seed=2)
            opt = ops.AdamW(net.masters, net.grads, lr=1e-3, copies=net.params)
            tokens, labels = (t.clone() for t in data[0])
            before = [p.clone() for p in net.masters]
            net.loss(tokens, labels)          # (buffers and libraries are there before the capture)
            torch.cuda.synchronize()
            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    loss = net.loss(tokens, labels)
                    opt.step(1)
            losses = []
            for t, y in data:
                tokens.copy_(t)
                labels.copy_(y)
                if captured:
                    graph.replay()
                    losses.append(loss.clone())
                else:
                    losses.append(net.loss(tokens, labels))
                    opt.step(1)
                torch.cuda.synchronize()
        results.append((losses, net.masters, net.grads))
        assert not any(torch.equal(a, b) for a, b in zip(before, net.masters))
    for a, b in zip(*results):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
