"""The loss of a last layer in several pieces of the classes; next to the two operators that it is made of; rows far apart; a logit past float32; what its
means and gradients are divided by.  Tolerances as in test_gpu_linear_xent.py, which checks against the definitions in 64 bits."""
import math

import pytest
import torch

from common_loss_shapes import PIECES
from paper_2012_15469_amd import ops
from test_gpu_linear_xent import DT, E, check, definition, half_step, near, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,k,classes,pad", PIECES)
def test_pieces(dtype, rows, k, classes, pad):
    x, w, labels, b = problem(rows, k, classes, dtype, 31, pad, ignored=0.1, masked=0.1)
    first = check(x, w, labels, b, smoothing=0.1, scale=16.0)
    again = ops.linear_cross_entropy(x, w, labels, b, smoothing=0.1, scale=16.0)
    assert all(torch.equal(a, c) for a, c in zip(first, again))
    del again
    # in a workspace with NaN in it: the first piece of dx is written, not added to
    a = dict(smoothing=0.1, scale=16.0, workspace=torch.full((3 << 28,), 255, dtype=torch.uint8, device="cuda"))
    again = ops.linear_cross_entropy(x, w, labels, b, **a)
    assert all(torch.equal(p, c) for p, c in zip(first, again))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,classes", [(300, 200, 1500), (7, 64, 20000), (2000, 80, 30000)])
def test_next_to_the_two_operators_apart(rows, k, classes, dtype):
    """linear_forward rounds logits to their type, h |z| each (h half a step), so losses differ by at most 2 h max |z| besides both sides' own errors, and p by
    p (2 h max |z|); cross_entropy rounds its gradient to that type, as this operator rounds its signal: h |g| on either side.  The products pass these on
    as sums of magnitudes."""
    x, w, labels, b = problem(rows, k, classes, dtype, 5, ignored=0.1)
    h = half_step(DT[dtype])
    z, _ = ops.linear_forward(x, w, b)
    mean1, loss1, g1 = ops.cross_entropy(z, labels)
    mean2, loss2, dx2, dw2, db2 = ops.linear_cross_entropy(x, w, labels, b)
    _, g, e_g, e_loss, count = definition(x, w, labels, b, 0.0, -100, 1.0)
    z64 = x.double() @ w.double() + b.double()
    dz = h * z64.abs().amax(1, keepdim=True)
    near(loss2, loss1.double(), 2 * e_loss + 2 * dz[:, 0], "loss")
    near(mean2, mean1.double(), float((2 * e_loss + 2 * dz[:, 0]).sum()) / count, "mean")
    used = (labels != -100).double()[:, None] / count
    e_two = 2 * e_g + 2 * dz * torch.softmax(z64, 1) * used + 2 * h * (g.abs() + e_g)
    dx1, dw1, db1 = ops.linear_backward(g1, x, w)
    x64, w64 = x.double(), w.double()
    near(dx2, dx1.double(), e_two @ w64.abs().t() + 2 * (classes + 2) * E * (g.abs() @ w64.abs().t()) + h * dx1.double().abs(), "dx")
    near(dw2, dw1.double(), x64.abs().t() @ e_two + 2 * (rows + 2) * E * (x64.abs().t() @ g.abs()) + h * dw1.double().abs(), "dw")
    near(db2, db1.double(), e_two.sum(0) + 2 * (rows + 2) * E * g.abs().sum(0) + h * db1.double().abs(), "db")


@pytest.mark.parametrize("rows,classes", [(6, 700), (6, 20000), (70, 5000), (4100, 17000)])
def test_a_logit_that_overflows(rows, classes):
    """A product past float32 makes a logit -inf: without smoothing its row's loss is that of the other classes, in whichever way the statistics are formed,
    and the class's part of the gradients is zero."""
    x, w, labels, b = problem(rows, 16, classes, "f32", 13)
    w[0], x[:, 0] = 0.0, 0.0
    labels.fill_(1)
    without = b.clone()
    without[3] = -math.inf
    loss_all, g_all, e_g, e_all, _ = definition(x, w, labels, b, 0.0, -100, 1.0)
    loss_two, g_two, e_g_two, e_two, _ = definition(x[2:3], w, labels[2:3], without, 0.0, -100, 1.0)
    loss_all[2], e_all[2], g_all[2], e_g[2] = loss_two[0], e_two[0], g_two[0] / rows, e_g_two[0] / rows
    w[0, 3], x[2, 0] = -10.0, 3e38
    for grads in (False, True):
        mean, loss, dx, dw, db = ops.linear_cross_entropy(x, w, labels, b, need_dx=grads, need_dw=grads, need_db=grads)
        near(loss, loss_all, e_all, "loss")
    near(db, g_all.sum(0), e_g.sum(0) + (rows + 2) * E * g_all.abs().sum(0), "db")
    assert float(dx[2, 0]) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(40, 300), (6, 20000), (3000, 17001)])
def test_what_it_is_divided_by(rows, classes, dtype):
    """Ignored rows count nowhere.  A row whose label is no class has loss NaN, and so has the mean, no gradient, and is one of those that the other rows'
    gradients are divided by, as for cross_entropy."""
    x, w, labels, b = problem(rows, 32, classes, dtype, 14)
    labels[0] = -100
    for bad in (classes, -1, classes + 5):
        labels[3] = bad
        for smoothing in (0.0, 0.1):
            mean, loss, dx, dw, db = check(x, w, labels, b, smoothing=smoothing)
            assert math.isnan(float(mean)) and math.isnan(float(loss[3])) and not math.isnan(float(loss[:3].sum() + loss[4:].sum())) and not dx[0].any() and not dx[3].any()
            there = ops.cross_entropy(ops.linear_forward(x, w, b)[0], labels, smoothing=smoothing)
            assert math.isnan(float(there[0])) and torch.equal(torch.isnan(there[1]), torch.isnan(loss)) and not there[2][3].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [1000, 20003])
def test_rows_far_apart(classes, dtype):
    """Rows more than 4 GB apart, in every table."""
    apart = ((1 << 31) + 64) // (2 if dtype == "f32" else 1)
    base = torch.empty(2 * apart + classes, dtype=DT[dtype], device="cuda")
    near_x, near_w, labels, b = problem(3, 3, classes, dtype, 15)
    labels[1] = -100
    want = ops.linear_cross_entropy(near_x, near_w, labels, b, smoothing=0.1)
    far_x, far_w = (base.as_strided((3, n), (apart, 1), at) for n, at in ((3, 0), (classes, 0)))
    far_x.copy_(near_x)
    check(far_x, near_w, labels, b, smoothing=0.1)
    far_w.copy_(near_w)
    check(near_x, far_w, labels, b, smoothing=0.1)
    for name, n in (("dx", 3), ("dw", classes)):
        out = base.as_strided((3, n), (apart, 1))
        out.fill_(7.0)
        got = ops.linear_cross_entropy(near_x, near_w, labels, b, smoothing=0.1, **{name: out})
        assert all(torch.equal(p, q) for p, q in zip(got, want)) and got[2 if name == "dx" else 3] is out
