"""Softmax cross-entropy and its gradient against the definition in 64 bits.

Tolerances: exponentials are taken of float32 differences, off by |z| 2^-22 and a few 2^-23, and a sum of n of them by at most n 2^-24 more, of
which lanes and wavefronts leave n / 64; the loss is a difference of values of size |z|.  So 2^-20 + n 2^-29 times (1 + max |z|), relative for the
gradient's probabilities, absolute for the loss, and 2^-8 of a bf16 gradient."""
import math

import pytest
import torch

from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def definition(z, labels, smoothing, ignore, scale):
    z = z.double()
    n = z.shape[1]
    left = ~(z == -math.inf)
    n_left = left.sum(1, keepdim=True).double()
    lse = torch.logsumexp(z, 1, keepdim=True)
    used = labels != ignore
    at = labels.clamp(0, n - 1).long()[:, None]
    hot = torch.zeros_like(z).scatter_(1, at, 1.0)
    target = (1 - smoothing) * hot + smoothing * left.double() / n_left
    loss = lse[:, 0] - (1 - smoothing) * z.gather(1, at)[:, 0] - smoothing * torch.where(left, z, 0.0).sum(1) / n_left[:, 0]
    if not smoothing:
        loss = lse[:, 0] - z.gather(1, at)[:, 0]
        target = hot
    p = torch.exp(z - lse)
    none = n_left[:, 0] == 0
    loss = torch.where(none, math.inf, loss)
    grad = torch.where(none[:, None], 0.0, p - target)
    known = (labels >= 0) & (labels < n)
    loss = torch.where(used, torch.where(known, loss, math.nan), 0.0)
    count = max(1, int(used.sum()))
    grad = torch.where((used & known)[:, None], grad, 0.0) * (scale / count)
    return loss.sum() / count, loss, grad, torch.where((used & ~none)[:, None], p, 0.0) * (scale / count), count


def check(z, labels, smoothing=0.0, ignore=-100, scale=1.0, size=None):
    n = z.shape[1]
    mean, loss, grad = ops.cross_entropy(z, labels, smoothing=smoothing, ignore_index=ignore, scale=scale)
    m, l, g, p, count = definition(z, labels, smoothing, ignore, scale)
    top = float(torch.where(torch.isfinite(z), z, 0.0).abs().max()) if z.numel() else 0.0
    tol = (2.0 ** -20 + n * 2.0 ** -29) * (1 + top)
    assert torch.equal(torch.isfinite(loss), torch.isfinite(l)) and torch.equal(torch.isnan(loss), torch.isnan(l))
    fine = torch.isfinite(l)
    assert float((loss.double() - l)[fine].abs().max() if fine.any() else 0.0) <= tol
    if torch.isfinite(m):
        assert abs(float(mean) - float(m)) <= tol
    else:
        assert float(mean) == float(m) or (math.isnan(float(mean)) and math.isnan(float(m)))
    limit = tol * p + (2.0 ** -8 if z.dtype == torch.bfloat16 else 2.0 ** -22) * g.abs() + 2.0 ** -22 * abs(scale) / count * (g != 0) + 1e-38
    ok = torch.isfinite(g)
    assert torch.equal(ok, torch.isfinite(grad))
    assert float(((grad.double() - g).abs() / limit)[ok].max() if ok.any() else 0.0) <= 1.0
    return mean, loss, grad


CLASSES = [1, 2, 7, 10, 64, 127, 128, 129, 500, 513, 1001, 2048, 2049, 4000, 8193, 20011, 32769, 50001, 66000, 131073]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", CLASSES)
def test_against_definition(n, dtype):
    gen = torch.Generator(device="cuda"); gen.manual_seed(n)
    for rows, smoothing, pad, shift, scale, bits in ((1, 0.0, 0, 0, 1.0, torch.int64), (19, 0.1, 3, 1, 128.0, torch.int32), (70, 0.3, 8, 0, 1.0, torch.int64)):
        wide = (3 * torch.randn(rows, n + pad + shift, generator=gen, device="cuda")).to(DT[dtype])
        z = wide[:, shift:shift + n]
        labels = torch.randint(n, (rows,), generator=gen, device="cuda").to(bits)
        if rows > 1:
            labels[::5] = -100
        if n > 2:
            out = torch.rand(rows, n, generator=gen, device="cuda") < 0.2
            out &= torch.arange(n, device="cuda") != labels[:, None]
            z.masked_fill_(out, -math.inf)
        _, _, grad = check(z, labels, smoothing, -100, scale)
        # in the place of the logits
        g2 = ops.cross_entropy(z, labels, smoothing=smoothing, scale=scale, grad=z)[2]
        assert g2 is z and torch.equal(g2, grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5, 200, 3000, 40000])
def test_rows_where_it_can_go_wrong(n, dtype):
    z = torch.randn(12, n, device="cuda").to(DT[dtype])
    labels = torch.arange(12, device="cuda") % n
    z[0] = -math.inf                                   # no class left
    z[1] = -math.inf; z[1, 1] = 2.0                    # only the label left
    z[2, 2] = -math.inf                                # the label ruled out
    z[3] = torch.finfo(z.dtype).min                    # a mask of the type's lowest value in every class
    z[4] = torch.finfo(z.dtype).min; z[4, 0] = 1.0
    z[5] = 80.0 * (torch.arange(n, device="cuda") % 3 - 1)
    z[6] = 3e4
    z[7, 0] = math.nan
    z[8, 0] = math.inf
    labels[9] = -100
    labels[10] = n                                     # not a class
    labels[11] = -5
    mean, loss, grad = ops.cross_entropy(z, labels)
    assert loss[0] == math.inf and not grad[0].float().any()
    assert float(loss[1]) == 0.0 and not grad[1].float().any()
    assert loss[2] == math.inf and torch.isfinite(grad[2]).all() and abs(float(grad[2, 2]) * 11 + 1) < 0.01
    assert abs(float(loss[3]) - math.log(n)) <= 1e-5 * math.log(n) and torch.isfinite(grad[3]).all()
    assert float(loss[4]) > 1e38 and abs(float(grad[4, 0]) * 11 - 1) < 0.01 and abs(float(grad[4, 4 % n]) * 11 + 1) < 0.01
    smooth = ops.cross_entropy(z[3:5], labels[3:5], smoothing=0.1)
    assert abs(float(smooth[1][0]) - math.log(n)) <= 1e-5 * math.log(n) and torch.isfinite(smooth[1]).all() and torch.isfinite(smooth[2]).all()
    assert float(loss[5]) >= 0 and torch.isfinite(grad[5]).all() and abs(float(loss[6]) - math.log(n)) <= 2.0 ** -20 * 3e4
    assert torch.isnan(loss[7]) and torch.isnan(grad[7]).all() and torch.isnan(loss[8]) and torch.isnan(grad[8, 0])
    assert float(loss[9]) == 0.0 and not grad[9].float().any()
    assert torch.isnan(loss[10]) and torch.isnan(loss[11]) and not grad[10:].float().any() and torch.isnan(mean)


def test_nothing_counts():
    for rows in (0, 5):
        z, labels = torch.randn(rows, 33, device="cuda"), torch.full((rows,), 7, device="cuda")
        mean, loss, grad = ops.cross_entropy(z, labels, ignore_index=7)
        assert float(mean) == 0.0 and loss.shape == (rows,) and not loss.any() and not grad.any()


def test_only_the_loss():
    z, labels = torch.randn(300, 1000, device="cuda"), torch.randint(1000, (300,), device="cuda")
    mean, loss, grad = ops.cross_entropy(z, labels, need_grad=False)
    m, l, _ = ops.cross_entropy(z, labels)
    assert grad is None and torch.equal(mean, m) and torch.equal(loss, l)


def test_gradient_against_differences():
    """Central differences of the definition in 64 bits (step 1e-4: their error is below 1e-8)."""
    z, labels, h = torch.randn(3, 9, device="cuda"), torch.tensor([1, -100, 8], device="cuda"), 1e-4
    z[0, 4] = -math.inf
    grad = ops.cross_entropy(z, labels, smoothing=0.2, scale=3.0)[2]
    for i in range(3):
        for j in range(9):
            hi, lo = z.double().clone(), z.double().clone()
            hi[i, j] += h
            lo[i, j] -= h
            want = float(definition(hi, labels, 0.2, -100, 3.0)[0] - definition(lo, labels, 0.2, -100, 3.0)[0]) * 3.0 / (2 * h)
            assert abs(float(grad[i, j]) - want) < 1e-5


def test_graph_replays():
    z, labels = torch.randn(200, 700, device="cuda").to(torch.bfloat16), torch.randint(700, (200,), device="cuda")
    ops.cross_entropy(z, labels)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.cross_entropy(z, labels, smoothing=0.1)
    for _ in range(3):
        z.copy_(torch.randn(200, 700, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ops.cross_entropy(z, labels, smoothing=0.1)))
