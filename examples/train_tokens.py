"""A network over a vocabulary trained by AdamW with the library's operators: embedding, layer norm, layers, and a loss whose logits are never in memory.

    python examples/train_tokens.py [--steps 200] [--vocab 5000] [--width 256]

It predicts each token of synthetic sequences from the `context` tokens before it: the rows of an embedding table, scaled by the root of their width, side by side; a layer to the network's
width; `blocks` residual blocks, each layer norm and a layer; layer norm; and the loss of the last layer's product.  The sequences follow a random table that says which few tokens may come behind
each, so there is something to learn.  Float32 masters, bf16 copies that AdamW writes for the operators, gradients written into the same buffers every step.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2012_15469_amd import ops  # noqa: E402


class TokenNetwork:
    """params: the embedding; the first layer's weight and bias; of each block the norm's weight and bias and the layer's; the last norm's; the last layer's."""

    def __init__(self, vocab, width, context=2, blocks=2, seed=0, device="cuda"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.vocab, self.width, self.context, self.blocks, self.scale = vocab, width, context, blocks, math.sqrt(width)

        def layer(k, n):
            return [torch.randn(k, n, generator=gen, device=device) / math.sqrt(k), torch.zeros(n, device=device)]

        def norm():
            return [torch.ones(width, device=device), torch.zeros(width, device=device)]

        self.masters = [torch.randn(vocab, width, generator=gen, device=device) / math.sqrt(width)] + layer(context * width, width)
        for _ in range(blocks):
            self.masters += norm() + layer(width, width)
        self.masters += norm() + layer(width, vocab)
        self.params = [p.to(torch.bfloat16) for p in self.masters]        # what the operators read
        self.grads = [torch.empty_like(p) for p in self.params]           # what they write
        self.decay = [0.01 if p.dim() > 1 else 0.0 for p in self.masters]

    def forward(self, tokens):
        """tokens [rows, context] -> the last norm's output, and what the backward pass needs."""
        p = self.params
        e = ops.embedding_forward(tokens.reshape(-1), p[0], scale=self.scale).view(tokens.shape[0], -1)
        x, pre = ops.linear_forward(e, p[1], p[2], act="gelu", keep_pre=True)
        kept = [(e, pre)]
        for b in range(self.blocks):
            g, s, w, bias = p[3 + 4 * b:7 + 4 * b]
            n, mean, rstd = ops.layer_norm_forward(x, g, s, keep_stats=True)
            y, pre = ops.linear_forward(n, w, bias, residual=x, act="gelu", keep_pre=True)
            kept.append((x, mean, rstd, n, pre))
            x = y
        h, mean, rstd = ops.layer_norm_forward(x, p[-4], p[-3], keep_stats=True)
        return h, kept + [(x, mean, rstd)]

    def loss(self, tokens, labels, *, smoothing=0.0, ignore_index=-100):
        """The mean loss; the gradients are in `grads`."""
        p, g = self.params, self.grads
        h, kept = self.forward(tokens)
        mean_loss, _, dh, _, _ = ops.linear_cross_entropy(h, p[-2], labels, p[-1], smoothing=smoothing, ignore_index=ignore_index, dw=g[-2], db=g[-1])
        x, mean, rstd = kept.pop()
        dy, _, _ = ops.layer_norm_backward(dh, x, mean, rstd, p[-4], dx=dh, dw=g[-4], db=g[-3])
        for b in reversed(range(self.blocks)):
            x, mean, rstd, n, pre = kept.pop()
            at = 3 + 4 * b
            dn, _, _ = ops.linear_backward(dy, n, p[at + 2], pre=pre, act="gelu", dw=g[at + 2], db=g[at + 3])
            dy, _, _ = ops.layer_norm_backward(dn, x, mean, rstd, p[at], residual=dy, dx=dn, dw=g[at], db=g[at + 1])
        e, pre = kept.pop()
        de, _, _ = ops.linear_backward(dy, e, p[1], pre=pre, act="gelu", dw=g[1], db=g[2])
        ops.embedding_backward(de.view(-1, self.width), tokens.reshape(-1), self.vocab, scale=self.scale, dw=g[0])
        return mean_loss

    def answer(self, tokens):
        """The most likely next token of each row."""
        return ops.linear_forward(self.forward(tokens)[0], self.params[-2], self.params[-1])[0].argmax(1)


def sequences(vocab, rows, length, seed=0, choices=4, device="cuda"):
    """Tokens of a chain: behind each token one of `choices`, the first of them half of the time."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    behind = torch.randint(vocab, (vocab, choices), generator=gen, device=device)
    out = [torch.randint(vocab, (rows,), generator=gen, device=device)]
    for _ in range(length - 1):
        which = (torch.randint(2, (rows,), generator=gen, device=device) * torch.randint(choices, (rows,), generator=gen, device=device))
        out.append(behind[out[-1], which])
    return torch.stack(out, 1)


def batches(data, context, rows, seed=0):
    """Without end: the tokens before a place of each of `rows` sequences, and the token there."""
    gen = torch.Generator(device=data.device)
    gen.manual_seed(seed)
    while True:
        r = torch.randint(data.shape[0], (rows, 1), generator=gen, device=data.device)
        at = torch.randint(context, data.shape[1], (rows, 1), generator=gen, device=data.device)
        yield data[r, at + torch.arange(-context, 0, device=data.device)], data[r[:, 0], at[:, 0]]


def train(steps, *, vocab=5000, width=256, context=2, blocks=2, rows=2048, lr=2e-3, state_bits=32, seed=0, report=None):
    """Trains for `steps` batches; returns the losses, the network and its optimiser."""
    net = TokenNetwork(vocab, width, context, blocks, seed)
    opt = ops.AdamW(net.masters, net.grads, lr=lr, weight_decay=net.decay, max_norm=1.0, state_bits=state_bits, copies=net.params)
    losses, batch = [], batches(sequences(vocab, 4096, 64, seed), context, rows, seed + 1)
    for k in range(steps):
        losses.append(net.loss(*next(batch)))
        opt.step()
        if report and (k + 1) % report == 0:
            print("step %4d  loss %.4f  gradient norm %.3f" % (k + 1, float(losses[-1]), float(opt.norm)), flush=True)
    return torch.stack(losses), net, opt


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--vocab", type=int, default=5000)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--rows", type=int, default=2048)
    ap.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    a = ap.parse_args()
    began = time.perf_counter()
    losses, net, opt = train(a.steps, vocab=a.vocab, width=a.width, rows=a.rows, state_bits=a.state_bits, report=max(1, a.steps // 10))
    torch.cuda.synchronize()
    print("%d parameters, %d steps of %d rows: loss %.4f -> %.4f (%.1f s with the data)" % (
        sum(p.numel() for p in net.masters), a.steps, a.rows, float(losses[0]), float(losses[-10:].mean()), time.perf_counter() - began))
    # one place answered: each operator's form for a single row
    print("behind tokens 1, 2:", int(net.answer(torch.tensor([[1, 2]], device="cuda"))))


if __name__ == "__main__":
    main()
