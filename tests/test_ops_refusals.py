"""Invalid arguments of the operators are refused on the host, before anything touches a device."""
import ctypes as C

import pytest
import torch

from common_ops import cada_linear, cada_linear_grad, cada_xent
from paper_2012_15469_amd import ops
from paper_2012_15469_amd.binding import _lib, cada_last_error

FAKE = 1 << 20          # an aligned address that nobody reads


LONG = dict(rows=64, in_=100000, ldx=100000)          # few tiles of a long contraction: split, with its parts in a workspace


def linear(**kw):
    a = cada_linear()
    a.rows, a.in_, a.out, a.type, a.act = 4, 8, 16, 1, 0
    a.x, a.ldx, a.w, a.ldw, a.y, a.ldy, a.workspace, a.workspace_bytes = FAKE, 8, FAKE, 16, FAKE, 16, FAKE, 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code,text", [
    (dict(rows=-1), -1, "rows"), (dict(in_=0), -1, "in and out"), (dict(out=1 << 25), -1, "in and out"), (dict(type=2), -1, "type"), (dict(act=4), -1, "act"),
    (dict(x=None), -1, "x is NULL"), (dict(ldx=7), -1, "row length of x"), (dict(ldw=15), -1, "row length of w"), (dict(y=None), -1, "y is NULL"), (dict(ldy=3), -1, "row length of y"),
    (dict(x=FAKE + 1), -1, "not aligned"), (dict(residual=FAKE, ldr=2), -1, "row length of residual"), (dict(pre=FAKE, ldpre=2), -1, "row length of pre"), (dict(bias=FAKE + 1), -1, "bias"),
    (dict(workspace=None, **LONG), -2, "workspace is NULL"), (dict(workspace=FAKE + 16, **LONG), -2, "256-byte"), (dict(workspace_bytes=1, **LONG), -2, "too small"), (dict(rows=1 << 40, in_=1 << 20, out=1 << 24), -1, "tiles")])
def test_linear_forward(kw, code, text):
    assert _lib.cada_linear_forward(C.byref(linear(**kw))) == code and text in cada_last_error()


@pytest.mark.parametrize("kw,code,text", [
    (dict(rows=-1), -1, "rows"), (dict(type=5), -1, "type"), (dict(act=-1), -1, "act"), (dict(dy=None), -1, "dy is NULL"), (dict(lddy=1), -1, "row length of dy"), (dict(act=1), -1, "pre is NULL"),
    (dict(x=None), -1, "x is NULL"), (dict(w=None), -1, "w is NULL"), (dict(lddx=1), -1, "row length of dx"), (dict(lddw=1), -1, "row length of dw"), (dict(db=FAKE + 1), -1, "db"),
    (dict(rows=100000, workspace_bytes=0), -2, "too small")])
def test_linear_backward(kw, code, text):
    a = cada_linear_grad()
    a.rows, a.in_, a.out, a.type, a.act = 4, 8, 16, 1, 0
    a.dy, a.lddy, a.x, a.ldx, a.w, a.ldw, a.dx, a.lddx, a.dw, a.lddw, a.db = FAKE, 16, FAKE, 8, FAKE, 16, FAKE, 8, FAKE, 16, FAKE
    a.workspace, a.workspace_bytes = FAKE, 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    assert _lib.cada_linear_backward(C.byref(a)) == code and text in cada_last_error()


@pytest.mark.parametrize("kw,code,text", [
    (dict(rows=-1), -1, "rows"), (dict(classes=0), -1, "classes"), (dict(classes=1 << 31), -1, "classes"), (dict(type=2), -1, "type"), (dict(label_bytes=2), -1, "label_bytes"),
    (dict(smoothing=1.0), -1, "smoothing"), (dict(smoothing=float("nan")), -1, "smoothing"), (dict(logits=None), -1, "device pointers"), (dict(labels=None), -1, "device pointers"),
    (dict(ldz=9), -1, "row length"), (dict(ldg=9), -1, "row length"), (dict(ldg=12, grad=FAKE), -1, "in the place"), (dict(labels=FAKE + 4), -1, "not aligned"), (dict(workspace=None), -2, "NULL")])
def test_cross_entropy(kw, code, text):
    a = cada_xent()
    a.rows, a.classes, a.type, a.label_bytes, a.logits, a.ldz, a.labels, a.grad, a.ldg = 1000, 10, 0, 8, FAKE, 10, FAKE, FAKE + 4096, 10
    a.workspace, a.workspace_bytes = FAKE, 1 << 20
    for k, v in kw.items():
        setattr(a, k, v)
    assert _lib.cada_cross_entropy(C.byref(a)) == code and text in cada_last_error()


@pytest.mark.parametrize("kw,tensor,code,text", [
    (dict(n_tensors=0), {}, -1, "tensors"), (dict(moment_bits=16), {}, -1, "moment_bits"), (dict(beta1=1.0), {}, -1, "beta"), (dict(beta2=-0.1), {}, -1, "beta"), (dict(eps=-1.0), {}, -1, "eps"),
    (dict(max_norm=-1.0), {}, -1, "max_norm"), (dict(max_norm=float("nan")), {}, -1, "max_norm"), (dict(m=None), {}, -1, "m and v"), (dict(v=FAKE + 4), {}, -1, "16-byte"),
    (dict(moment_bits=8), {}, -1, "m_scale"), ({}, dict(n=-1), -1, "n must be"), ({}, dict(param=None), -1, "param and grad"), ({}, dict(param_type=3), -1, "types"),
    ({}, dict(grad=FAKE + 2), -1, "not aligned"), ({}, dict(weight_decay=float("inf")), -1, "weight_decay"), (dict(workspace_bytes=16), {}, -2, "too small")])
def test_adamw(kw, tensor, code, text):
    t = (ops.cada_adamw_tensor * 1)()
    t[0].param, t[0].grad, t[0].n = FAKE, FAKE, 100
    cfg = ops.cada_adamw_config()
    cfg.tensors, cfg.n_tensors, cfg.moment_bits, cfg.m, cfg.v, cfg.beta1, cfg.beta2, cfg.eps = t, 1, 32, FAKE, FAKE, 0.9, 0.999, 1e-8
    cfg.workspace, cfg.workspace_bytes = FAKE, 1 << 20
    for k, v in kw.items():
        setattr(cfg, k, v)
    for k, v in tensor.items():
        setattr(t[0], k, v)
    out = C.c_void_p(5)
    assert _lib.cada_adamw_init(C.byref(cfg), C.byref(out)) == code and text in cada_last_error() and out.value is None


def test_null_arguments():
    assert _lib.cada_linear_forward(None) == -1 and _lib.cada_linear_backward(None) == -1 and _lib.cada_cross_entropy(None) == -1
    assert _lib.cada_linear_forward_workspace(None) == -1 and _lib.cada_linear_backward_workspace(None) == -1 and _lib.cada_xent_workspace(None) == -1
    assert _lib.cada_adamw_init(None, None) == -1 and _lib.cada_adamw_step(None, 1, 1e-3, None) == -1 and _lib.cada_adamw_moments(None, None, None) == -1
    assert _lib.cada_adamw_moment_elements(None) == -1 and _lib.cada_adamw_workspace(None) == -1
    _lib.cada_adamw_destroy(None)


def test_sizes_without_gpu():
    t = (ops.cada_adamw_tensor * 3)()
    for x, n in zip(t, (1, 256, 257)):
        x.n = n
    cfg = ops.cada_adamw_config()
    cfg.tensors, cfg.n_tensors = t, 3
    assert _lib.cada_adamw_moment_elements(C.byref(cfg)) == 256 + 256 + 512
    assert _lib.cada_adamw_workspace(C.byref(cfg)) == 0 and cfg.workspace_bytes >= 3 * 40
    a = linear(rows=0, workspace=None)
    assert _lib.cada_linear_forward_workspace(C.byref(a)) == 0 and a.workspace_bytes == 0
    assert _lib.cada_linear_forward(C.byref(a)) == 0          # nothing to do


@pytest.mark.parametrize("call,text", [
    (lambda x: ops.linear_forward(x, x), "GPU"), (lambda x: ops.linear_backward(x, x, x), "GPU"), (lambda x: ops.cross_entropy(x, x), "GPU"),
    (lambda x: ops.AdamW([x], [x]), "GPU"), (lambda x: ops.AdamW([x], []), "one length"), (lambda x: ops.AdamW([x], [x], state_bits=4), "32 or 8"),
    (lambda x: ops.AdamW([x], [x], weight_decay=[0.1, 0.2]), "one value")])
def test_tensors_that_are_not_on_a_gpu(call, text):
    with pytest.raises(ValueError, match=text):
        call(torch.zeros(4, 4))


MB = 1 << 20


@pytest.mark.parametrize("kw,text", [
    (dict(y=1 * MB), "y and x"), (dict(y=2 * MB), "y and w"), (dict(y=2 * MB + 8 * 32 - 2), "y and w"), (dict(bias=3 * MB + 32), "y and bias"), (dict(pre=3 * MB, ldpre=16), "y and pre"),
    (dict(pre=1 * MB, ldpre=16), "pre and x"), (dict(residual=3 * MB + 2, ldr=16), "y and residual"), (dict(residual=3 * MB, ldr=17), "y and residual"),
    (dict(pre=5 * MB, ldpre=16, residual=5 * MB, ldr=16), "pre and residual"), (dict(y=1 * MB + 14, ldy=24, ldx=24), "y and x"), (dict(y=1 * MB + 18, ldy=24, ldx=24), "y and x")])
def test_linear_forward_in_place(kw, text):
    a = linear(**{**dict(x=1 * MB, w=2 * MB, y=3 * MB), **kw})
    assert _lib.cada_linear_forward(C.byref(a)) == -1 and text + " share memory" in cada_last_error()


@pytest.mark.parametrize("kw,text", [
    (dict(dx=1 * MB), "dx and dy"), (dict(dw=2 * MB), "dw and x"), (dict(dw=3 * MB), "dw and w"), (dict(db=1 * MB), "db and dy"), (dict(dx=3 * MB), "dx and w"), (dict(dx=7 * MB, lddx=8), "dx and pre"),
    (dict(dw=4 * MB), "dw and dx"), (dict(db=5 * MB + 8 * 32 - 2), "db and dw")])
def test_linear_backward_in_place(kw, text):
    a = cada_linear_grad()
    a.rows, a.in_, a.out, a.type, a.act = 4, 8, 16, 1, 1
    a.dy, a.lddy, a.x, a.ldx, a.w, a.ldw, a.dx, a.lddx, a.dw, a.lddw, a.db, a.pre, a.ldpre = 1 * MB, 16, 2 * MB, 8, 3 * MB, 16, 4 * MB, 8, 5 * MB, 16, 6 * MB, 7 * MB, 16
    a.workspace, a.workspace_bytes = 8 * MB, 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    assert _lib.cada_linear_backward(C.byref(a)) == -1 and text + " share memory" in cada_last_error()


def test_cross_entropy_partly_in_place():
    a = cada_xent()
    a.rows, a.classes, a.type, a.label_bytes, a.logits, a.ldz, a.labels, a.grad, a.ldg = 1000, 10, 0, 8, MB, 10, 2 * MB, MB + 4, 10
    a.workspace, a.workspace_bytes = 4 * MB, 1 << 20
    assert _lib.cada_cross_entropy(C.byref(a)) == -1 and "grad and logits share memory" in cada_last_error()
