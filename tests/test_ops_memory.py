"""Operands and outputs that lie in one another's memory, by addresses that nobody reads: what is refused, and what is not (such a call carries another fault, which is then the one named)."""
import ctypes as C

import pytest

from common_ops import cada_linear, cada_linear_grad, cada_xent
from paper_2012_15469_amd import ops
from paper_2012_15469_amd.binding import _lib, cada_last_error

MB = 1 << 20


@pytest.mark.parametrize("y,bias,apart", [(0, 40, True), (0, 5 * 96 + 40, True), (0, 4 * 96 + 56, True), (0, 5 * 96 + 57, False), (0, 39, False), (0, 6 * 96, False), (40, 0, True), (40, 96, True), (40, 96 + 1, False), (40, 69 * 96 + 80, True)])
def test_a_single_row_beside_columns(y, bias, apart):
    """70 rows of 40 outputs, 96 elements apart, and a bias of 40 in one of the rows' remaining 56 elements, or not quite."""
    a = cada_linear()
    a.rows, a.in_, a.out, a.type, a.act = 70, 8, 40, 0, 0
    a.x, a.ldx, a.w, a.ldw, a.y, a.ldy, a.bias = MB, 8, 2 * MB, 40, 4 * MB + 4 * y, 96, 4 * MB + 4 * bias
    a.pre, a.ldpre, a.residual, a.ldr = 6 * MB, 40, 6 * MB, 40
    assert _lib.cada_linear_forward(C.byref(a)) == -1
    assert ("pre and residual" if apart else "y and bias") + " share memory" in cada_last_error()


def adamw(n=1000, bits=32, count=3, max_norm=0.0, **kw):
    """Three tensors whose parts lie one MB after the other; `kw` moves parts: "param2", "copy0", "m", ..."""
    t = (ops.cada_adamw_tensor * count)()
    for i in range(count):
        t[i].param, t[i].grad, t[i].copy, t[i].n = MB * (10 * i + 1), MB * (10 * i + 2), MB * (10 * i + 3), n
    cfg = ops.cada_adamw_config()
    cfg.tensors, cfg.n_tensors, cfg.moment_bits, cfg.beta1, cfg.beta2, cfg.eps, cfg.max_norm = t, count, bits, 0.9, 0.999, 1e-8, max_norm
    cfg.m, cfg.v, cfg.m_scale, cfg.v_scale, cfg.norm, cfg.workspace, cfg.workspace_bytes = (MB * i for i in (100, 101, 102, 103, 104, 105, 1))
    for k, v in kw.items():
        if k[-1].isdigit():
            setattr(t[int(k[-1])], k[:-1], v)
        else:
            setattr(cfg, k, v)
    out = C.c_void_p()
    rc = _lib.cada_adamw_init(C.byref(cfg), C.byref(out))
    assert rc == -1 and not out.value
    return cada_last_error()


@pytest.mark.parametrize("kw,text", [
    (dict(param1=1 * MB), "param 0 and param 1"), (dict(param2=1 * MB + 3996), "param 0 and param 2"), (dict(copy0=1 * MB), "0 and "), (dict(copy1=11 * MB + 3998), "param 1 and copy 1"),
    (dict(param0=2 * MB), "0 and "), (dict(grad2=1 * MB + 4), "param 0 and grad 2"), (dict(grad0=3 * MB), "0 and "), (dict(copy2=3 * MB), "0 and copy"), (dict(m=1 * MB), " and "), (dict(v=100 * MB + 3 * 4096 - 16), "m and v"),
    (dict(v=2 * MB + 16), "grad 0 and v"), (dict(workspace=23 * MB), " and "), (dict(norm=1 * MB + 8, max_norm=1.0), "param 0 and norm"), (dict(m_scale=100 * MB + 2048, bits=8), "m and m_scale"),
    (dict(v_scale=102 * MB + 44, bits=8), "m_scale and v_scale")])
def test_adamw(kw, text):
    error = adamw(**kw)
    assert "share memory" in error and text in error


def test_what_a_step_only_reads_or_does_not_touch_may_be_shared():
    """Gradients of several tensors, ends that meet, moments of 8 bits where 32 would not fit, a norm without clipping, parts of no elements: the fault that is named is the one planted last."""
    last = dict(param2=11 * MB)
    for kw in (dict(grad1=2 * MB, grad2=2 * MB + 4), dict(grad1=1 * MB + 4000), dict(v=100 * MB + 3 * 1024, bits=8), dict(norm=1 * MB), dict(m_scale=1 * MB, v_scale=1 * MB)):
        assert "param 1 and param 2 share memory" in adamw(**{**kw, **last}), kw
    assert "share memory" in adamw(n=1, param1=1 * MB)


@pytest.mark.parametrize("kw,text", [
    (dict(loss=1 * MB + 39996), "loss and logits"), (dict(mean=1 * MB), "mean and logits"), (dict(workspace=1 * MB - 256), "workspace and logits"), (dict(grad=2 * MB - 40000 + 4), "grad and labels"),
    (dict(loss=2 * MB), "loss and labels"), (dict(mean=2 * MB + 7996), "mean and labels"), (dict(loss=5 * MB), "loss and grad"), (dict(mean=6 * MB + 3996), "mean and loss"),
    (dict(mean=5 * MB + 16), "mean and grad"), (dict(workspace=2 * MB), "workspace and labels"), (dict(workspace=5 * MB), "workspace and grad"), (dict(workspace=6 * MB), "workspace and loss"),
    (dict(mean=8 * MB + 64), "workspace and mean"), (dict(loss=1 * MB + 40, ldz=10 + 999), "loss and logits"), (dict(labels=1 * MB, grad=1 * MB), "grad and labels"), (dict(rows=0, mean=8 * MB), "workspace and mean")])
def test_cross_entropy(kw, text):
    a = cada_xent()
    a.rows, a.classes, a.type, a.label_bytes, a.logits, a.ldz, a.labels, a.grad, a.ldg = 1000, 10, 0, 8, MB, 10, 2 * MB, 5 * MB, 10
    a.loss, a.mean, a.workspace, a.workspace_bytes = 6 * MB, 7 * MB, 8 * MB, 1 << 20
    for k, v in kw.items():
        setattr(a, k, v)
    assert _lib.cada_cross_entropy(C.byref(a)) == -1 and text + " share memory" in cada_last_error()


@pytest.mark.parametrize("part,cols", [("x", 4096), ("w", 10), ("bias", 10), ("y", 10), ("pre", 10), ("residual", 10)])
def test_workspace_of_a_layer(part, cols):
    """A long contraction, whose parts lie in the workspace."""
    a = cada_linear()
    a.rows, a.in_, a.out, a.type, a.act = 64, 4096, 10, 0, 0
    a.x, a.ldx, a.w, a.ldw, a.bias, a.y, a.ldy, a.pre, a.ldpre, a.residual, a.ldr = 10 * MB, 4096, 20 * MB, 10, 30 * MB, 40 * MB, 10, 50 * MB, 10, 60 * MB, 10
    a.workspace = 70 * MB
    assert _lib.cada_linear_forward_workspace(C.byref(a)) == 0 and 256 < a.workspace_bytes < MB
    setattr(a, part, a.workspace + a.workspace_bytes - 256)
    assert _lib.cada_linear_forward(C.byref(a)) == -1 and "workspace and %s share memory" % part in cada_last_error()


@pytest.mark.parametrize("part", ["dy", "x", "w", "pre", "dx", "dw", "db"])
def test_workspace_of_a_layers_gradients(part):
    a = cada_linear_grad()
    a.rows, a.in_, a.out, a.type, a.act = 512, 512, 512, 1, 1
    for i, name in enumerate(("dy", "x", "w", "pre", "dx", "dw")):
        setattr(a, name, 10 * (i + 1) * MB)
        setattr(a, "ld" + name, 512)
    a.db, a.workspace = 80 * MB, 90 * MB
    assert _lib.cada_linear_backward_workspace(C.byref(a)) == 0 and 512 * 512 * 2 < a.workspace_bytes < 10 * MB
    setattr(a, part, a.workspace + 1024)
    assert _lib.cada_linear_backward(C.byref(a)) == -1 and "workspace and %s share memory" % part in cada_last_error()


@pytest.mark.parametrize("rows,text", [(1, "mean and labels share memory"), (2, "must have their row length")])
def test_the_gradient_of_one_row_in_place(rows, text):
    """One row has no distance to a next one."""
    a = cada_xent()
    a.rows, a.classes, a.type, a.label_bytes, a.logits, a.ldz, a.labels, a.grad, a.ldg = rows, 10, 0, 8, MB, 10, 2 * MB, MB, 12
    a.mean, a.workspace, a.workspace_bytes = 2 * MB + 4, 8 * MB, 1 << 20
    assert _lib.cada_cross_entropy(C.byref(a)) == -1 and text in cada_last_error()
