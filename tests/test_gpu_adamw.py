"""The AdamW step against the formulas in 64 bits, and 8-bit codes against their definition.

Tolerances: an update is about ten float32 operations, 16 x 2^-24 of its terms; a bf16 parameter adds 2^-8 of itself.  8-bit codes and scales are the
definition's exactly where the float32 operations in the order of cada_ops.h are made by torch one by one."""
import math

import pytest
import torch

from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
BLOCK = 256
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [1, 7, 255, 256, 257, 2047, 2048, 2049, 5000, 70001, 0, 3]


def tensors(sizes, ptype, gtype, gen, scale=1e-2, shift=0):
    """Contiguous tensors, `shift` elements into their memory."""
    p = [torch.randn(n + shift, generator=gen, device="cuda").to(DT[ptype])[shift:] for n in sizes]
    g = [(scale * torch.randn(n + shift, generator=gen, device="cuda")).to(DT[gtype])[shift:] for n in sizes]
    return p, g


@pytest.mark.parametrize("clip", [0.0, 0.05])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")], ids=str)
def test_three_steps_of_32_bits(types, shift, clip):
    gen = torch.Generator(device="cuda"); gen.manual_seed(1)
    params, grads = tensors(SIZES, *types, gen, shift=shift)
    copies = [torch.empty_like(p, dtype=torch.bfloat16) if i % 2 else None for i, p in enumerate(params)]
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    lr, b1, b2, eps = 1e-2, 0.9, 0.99, 1e-8
    opt = ops.AdamW(params, grads, lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=decay, max_norm=clip, copies=copies)
    scale = torch.tensor([0.5], device="cuda")
    for t in (1, 2, 3):
        for g in grads:
            g.copy_(1e-2 * torch.randn(g.shape, generator=gen, device="cuda"))
        p0, (m0, v0) = [p.double() for p in params], [x.double() for x in opt.moments()]
        opt.step(grad_scale=scale if t == 2 else None)
        factor = 0.5 if t == 2 else 1.0
        norm = factor * math.sqrt(sum(float(g.double().square().sum()) for g in grads))
        if clip:
            assert abs(float(opt.norm) - norm) <= 1e-6 * norm
            factor *= min(1.0, clip / norm)
        m, v = opt.moments()
        for i, (p, g, at) in enumerate(zip(params, grads, opt.offsets)):
            n = p.numel()
            gd = g.double() * factor
            m1, v1 = b1 * m0[at:at + n] + (1 - b1) * gd, b2 * v0[at:at + n] + (1 - b2) * gd * gd
            assert ((m[at:at + n].double() - m1).abs() <= 8 * U * (m0[at:at + n].abs() + gd.abs())).all()
            assert ((v[at:at + n].double() - v1).abs() <= 8 * U * v1).all()
            end = at + -(-n // BLOCK) * BLOCK
            assert not m[at + n:end].any() and not v[at + n:end].any()
            up = lr * (m1 / (1 - b1 ** t)) / (torch.sqrt(v1 / (1 - b2 ** t)) + eps)
            want = p0[i] * (1 - lr * decay[i]) - up
            # (the update's error: that of m, of which it is a multiple, relative to the terms it was formed from)
            spread = lr / (1 - b1 ** t) * (m0[at:at + n].abs() + gd.abs()) / (torch.sqrt(v1 / (1 - b2 ** t)) + eps)
            limit = 16 * U * spread + 2 * U * p0[i].abs() + (2.0 ** -8 * want.abs() if types[0] == "bf16" else 0)
            assert ((p.double() - want).abs() <= limit).all()
            if copies[i] is not None and types[0] == "f32":
                assert torch.equal(copies[i], p.to(torch.bfloat16))


def encode(x, top, root):
    """The definition's codes and scales, operation by operation in float32."""
    b = torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)
    s = b.abs().amax(1)
    inv = torch.where(s >= 1e-30, torch.full_like(s, float(top * top)) / s, torch.zeros_like(s))
    q = torch.round(torch.sqrt(b.abs() * inv[:, None])).clamp(max=top)
    if root:
        return torch.where(b > 0, q.clamp(min=1), q).to(torch.uint8).view(-1), s
    return torch.where(b < 0, -q, q).to(torch.int8).view(-1), s


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16")], ids=str)
def test_8_bit_codes_are_the_definitions(types):
    gen = torch.Generator(device="cuda"); gen.manual_seed(2)
    params, grads = tensors(SIZES, *types, gen)
    b1, b2, lr, eps = 0.9, 0.999, 1e-3, 1e-8
    opt = ops.AdamW(params, grads, lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=0.01, state_bits=8)
    for t in range(1, 5):
        for i, g in enumerate(grads):
            size = 10.0 ** (3 * i % 11 - 5)
            g.copy_(size * torch.randn(g.shape, generator=gen, device="cuda") * torch.exp(2 * torch.randn(g.shape, generator=gen, device="cuda")))
            if g.numel() > 300:
                g[:40] = 0
        p0, (m0, v0) = [p.clone() for p in params], opt.moments()
        opt.step()
        m, v = opt.moments()
        for i, (p, g, at) in enumerate(zip(params, grads, opt.offsets)):
            n, end = p.numel(), at + -(-p.numel() // BLOCK) * BLOCK
            gf = g.float()
            m1 = m0[at:at + n] * b1 + gf * (1 - b1)
            v1 = v0[at:at + n] * b2 + (gf * (1 - b2)) * gf
            r1 = torch.sqrt(v1)
            for (codes, scales), x, top in ((opt.m, m1, 127), (opt.v, r1, 255)):
                q, s = encode(x, top, top == 255)
                assert torch.equal(scales[at // BLOCK:end // BLOCK], s) and torch.equal(codes[at:end], q)
            pf = p0[i].float()
            new = (pf - pf * (lr * 0.01)) - (m1 * (lr / (1 - b1 ** t))) / (r1 * (1 / math.sqrt(1 - b2 ** t)) + eps)
            assert torch.equal(p, new.to(p.dtype))
            # the values: q |q| s / 127^2 and (c^2 s / 255^2)^2
            q, c = opt.m[0][at:end].double(), opt.v[0][at:end].double()
            sm, sv = (s[1][at // BLOCK:end // BLOCK].double().repeat_interleave(BLOCK) for s in (opt.m, opt.v))
            assert torch.allclose(m[at:end].double(), q * q.abs() * sm / 127 ** 2, rtol=4 * U, atol=1e-37)
            assert torch.allclose(v[at:end].double(), (c * c * sv / 255 ** 2) ** 2, rtol=8 * U, atol=1e-37)
            # nothing that divides has become zero, and what was coded is near
            assert ((v[at:at + n] > 0) == (r1 * r1 > 0)).all() or float(r1[r1 > 0].min()) < 1e-18
            near = m1.abs() > 0.01 * m1.abs().max() if n else m1 > 0
            assert ((m[at:at + n] - m1).abs()[near] <= 0.13 * m1.abs()[near]).all()


def test_what_is_not_finite_is_not_hidden():
    for bits in (32, 8):
        params, grads = [torch.ones(1000, device="cuda"), torch.ones(300, device="cuda")], [torch.full((1000,), 0.1, device="cuda"), torch.full((300,), 0.1, device="cuda")]
        grads[0][700] = math.nan
        opt = ops.AdamW(params, grads, state_bits=bits)
        opt.step()
        m, v = opt.moments()
        assert torch.isnan(params[0][700]) and torch.isnan(m[700]) and torch.isnan(v[700])
        assert torch.isfinite(params[0][:700]).all() and torch.isfinite(params[1]).all() and torch.isfinite(m[1024:]).all() and torch.isfinite(m[:512]).all()
        clipped = ops.AdamW(params[1:], [grads[0][600:900]], state_bits=bits, max_norm=1.0)
        clipped.step()
        assert torch.isnan(clipped.norm) and torch.isnan(params[1]).all()


def test_zero_gradients_and_tiny_ones():
    for bits in (32, 8):
        params, grads = [torch.ones(600, device="cuda")], [torch.zeros(600, device="cuda")]
        opt = ops.AdamW(params, grads, lr=0.1, state_bits=bits, max_norm=1.0)
        opt.step()
        assert torch.equal(params[0], torch.ones(600, device="cuda")) and float(opt.norm) == 0.0
        grads[0].fill_(1e-32)
        opt.step()
        assert torch.isfinite(params[0]).all() and torch.isfinite(opt.moments()[1]).all()


def test_norm_of_large_gradients():
    """Squares that float32 does not hold."""
    params, grads = [torch.zeros(5000, device="cuda")], [torch.full((5000,), 1e25, device="cuda")]
    opt = ops.AdamW(params, grads, lr=0.1, max_norm=1.0)
    opt.step()
    want = 1e25 * math.sqrt(5000)
    assert abs(float(opt.norm) - want) < 1e-6 * want and torch.isfinite(params[0]).all() and float(params[0].abs().min()) > 0.05


def test_going_on_from_saved_moments_and_many_tensors():
    gen = torch.Generator(device="cuda"); gen.manual_seed(7)
    for bits in (32, 8):
        sizes = [int(x) for x in torch.randint(1, 3000, (300,), generator=gen, device="cuda").tolist()]
        params, grads = tensors(sizes, "f32", "f32", gen)
        other = [p.clone() for p in params]
        a = ops.AdamW(params, grads, lr=1e-2, state_bits=bits, max_norm=0.3)
        b = ops.AdamW(other, grads, lr=1e-2, state_bits=bits, max_norm=0.3)
        for _ in range(3):
            a.step()
        b.step()
        saved = tuple(tuple(x.clone() for x in s) for s in (b.m, b.v)) if bits == 8 else (b.m.clone(), b.v.clone())
        b.close()
        c = ops.AdamW(other, grads, lr=1e-2, state_bits=bits, max_norm=0.3, moments=saved)
        c.step(2)
        c.step()
        assert c.t == 3 and all(torch.equal(p, q) for p, q in zip(params, other))


def test_one_step_of_a_captured_graph():
    params, grads = [torch.ones(5000, device="cuda")], [torch.randn(5000, device="cuda")]
    other = [params[0].clone()]
    a, b = ops.AdamW(params, grads, max_norm=1.0, state_bits=8), ops.AdamW(other, grads, max_norm=1.0, state_bits=8)
    s = torch.cuda.Stream()
    a.close()
    a = ops.AdamW(params, grads, max_norm=1.0, state_bits=8, stream=s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        a.step(1)
    for _ in range(3):
        grads[0].copy_(torch.randn(5000, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        b.step(1)
        torch.cuda.synchronize()
        assert torch.equal(params[0], other[0])
