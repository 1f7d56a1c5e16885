"""A residual network trained by AdamW with the library's operators, next to the engine on the same data.

    python examples/train_network.py [--steps 200] [--state-bits 32|8] [--engine]

The data is workload 4's: 64 workers' samples of 784 features in ten classes, the workers' minibatches taken together as one batch (everybody uploads, which
is the baseline that CADA saves communication against).  The network is 784 -> width, `blocks` residual blocks of width, -> 10: float32
masters, bf16 copies that AdamW writes for the products, and gradients that the layers' backward passes write into the same buffers every
step, so a step allocates little and synchronises nothing.  --engine trains workload 4's own network with CADA2 for as many steps and prints its objective.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from cada_synth import configs, generators  # noqa: E402
from paper_2012_15469_amd import ops  # noqa: E402
from paper_2012_15469_amd.binding import Cada  # noqa: E402


class Network:
    """Layers y = act(x w + b) (+ x where the widths agree) and a last one without activation."""

    def __init__(self, widths, act="gelu", seed=0, device="cuda"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.act, n = act, len(widths) - 1
        self.residual = [widths[i] == widths[i + 1] and i < n - 1 for i in range(n)]
        self.acts = [act] * (n - 1) + ["none"]
        self.masters = []
        for k, m in zip(widths, widths[1:]):
            self.masters.append(torch.randn(k, m, generator=gen, device=device) / math.sqrt(k))
            self.masters.append(torch.zeros(m, device=device))
        self.params = [p.to(torch.bfloat16) for p in self.masters]        # what the products read
        self.grads = [torch.empty_like(p) for p in self.params]           # what they write
        self.decay = [0.01 if p.dim() > 1 else 0.0 for p in self.masters]

    def forward(self, x, keep=True):
        """Logits, and what the backward pass needs: each layer's input and pre-activation."""
        kept = []
        for i, act in enumerate(self.acts):
            y, pre = ops.linear_forward(x, self.params[2 * i], self.params[2 * i + 1], residual=x if self.residual[i] else None, act=act,
                                        keep_pre=keep and act != "none")
            kept.append((x, pre))
            x = y
        return x, kept

    def backward(self, dy, kept):
        for i in reversed(range(len(self.acts))):
            x, pre = kept[i]
            dx, _, _ = ops.linear_backward(dy, x, self.params[2 * i], pre=pre, act=self.acts[i], need_dx=i > 0, dw=self.grads[2 * i], db=self.grads[2 * i + 1])
            if i > 0 and self.residual[i]:
                dx.add_(dy)
            dy = dx


def batches(prob, sched, device):
    """Minibatch k of all workers as one batch: features bf16, labels."""
    X, y = torch.from_numpy(prob.X).to(device), torch.from_numpy(prob.y).to(device)
    M, rows = sched.shape[1], X.shape[0] // sched.shape[1]
    start = torch.arange(M, device=device)[:, None] * rows
    for idx in torch.from_numpy(sched).to(device):
        at = (start + idx).view(-1)
        yield X[at].to(torch.bfloat16), y[at]


def train(cfg, steps, *, width=512, blocks=2, lr=1e-3, state_bits=32, smoothing=0.0, seed=0, report=None):
    """Trains for `steps` batches; returns the losses, the network and its optimiser."""
    device = torch.device("cuda")
    prob, sched = generators.make_problem(cfg), generators.make_schedule(cfg, steps)
    net = Network([cfg.layer_dims[0]] + [width] * (blocks + 1) + [cfg.layer_dims[-1]], seed=seed)
    opt = ops.AdamW(net.masters, net.grads, lr=lr, weight_decay=net.decay, max_norm=1.0, state_bits=state_bits, copies=net.params)
    losses = []
    for k, (x, y) in enumerate(batches(prob, sched, device)):
        logits, kept = net.forward(x)
        loss, _, dlogits = ops.cross_entropy(logits, y, smoothing=smoothing, grad=logits)
        net.backward(dlogits, kept)
        opt.step()
        losses.append(loss)
        if report and (k + 1) % report == 0:
            print("step %4d  loss %.4f  gradient norm %.3f" % (k + 1, float(loss), float(opt.norm)), flush=True)
    return torch.stack(losses), net, opt


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    ap.add_argument("--engine", action="store_true", help="also train workload 4's own network with CADA2")
    a = ap.parse_args()
    cfg = configs.CFG4
    began = time.perf_counter()
    losses, net, opt = train(cfg, a.steps, width=a.width, blocks=a.blocks, state_bits=a.state_bits, report=max(1, a.steps // 10))
    torch.cuda.synchronize()
    print("%d parameters, %d steps of %d rows, moments in %d bits: loss %.4f -> %.4f (%.1f s with the data)" % (
        sum(p.numel() for p in net.masters), a.steps, cfg.M * cfg.B, a.state_bits, float(losses[0]), float(losses[-10:].mean()), time.perf_counter() - began))
    # one sample answered: the layers' form for a few rows
    x = torch.rand(1, cfg.layer_dims[0], device="cuda").to(torch.bfloat16)
    print("class of one sample:", int(net.forward(x, keep=False)[0].argmax()))
    if a.engine:
        prob, sched = generators.make_problem(cfg), generators.make_schedule(cfg, a.steps)
        eng = Cada.from_config(cfg, torch.from_numpy(prob.X).cuda(), torch.from_numpy(prob.y).cuda(), torch.from_numpy(prob.theta0).cuda())
        eng.run(torch.from_numpy(sched).cuda())
        out = eng.evaluate()
        torch.cuda.synchronize()
        uploads = int(eng.state()["uploads_total"])
        torch.cuda.synchronize()
        print("CADA2, %s: objective %.4f, accuracy %.3f, %d uploads of %d" % ("-".join(map(str, cfg.layer_dims)), float(out[0]), float(out[1]), uploads, a.steps * cfg.M))
        eng.close()


if __name__ == "__main__":
    main()
