"""Invalid arguments of layer norm and of the embedding are refused on the host, before anything touches a device; memory that is shared, by addresses that nobody reads."""
import ctypes as C

import pytest
import torch

from common_more_ops import cada_embedding, cada_embedding_grad, cada_norm, cada_norm_grad, filled
from paper_2012_15469_amd import ops
from paper_2012_15469_amd.binding import _lib, cada_last_error

MB = 1 << 20
NORM = dict(rows=10, width=16, type=1, eps=1e-5, x=1 * MB, ldx=16, weight=2 * MB, bias=3 * MB, y=4 * MB, ldy=16, mean=5 * MB, rstd=6 * MB)
NORM_GRAD = dict(rows=1000, width=16, type=1, dy=1 * MB, lddy=16, x=2 * MB, ldx=16, mean=3 * MB, rstd=4 * MB, weight=5 * MB, residual=6 * MB, ldr=16, dx=7 * MB, lddx=16, dw=8 * MB, db=9 * MB,
                 workspace=10 * MB, workspace_bytes=1 << 26)
EMBED = dict(rows=10, vocab=100, width=16, type=1, token_bytes=8, tokens=1 * MB, ignore_index=-100, w=2 * MB, ldw=16, scale=1.0, y=3 * MB, ldy=16)
EMBED_GRAD = dict(rows=1000, vocab=100, width=16, type=0, token_bytes=4, tokens=1 * MB, ignore_index=-100, dy=2 * MB, lddy=16, scale=1.0, dw=3 * MB, lddw=16, workspace=4 * MB, workspace_bytes=1 << 26)
SHARE = " share memory"


def refused(call, kind, base, kw, code, text):
    assert getattr(_lib, call)(C.byref(filled(kind, base, **kw))) == code and text in cada_last_error(), cada_last_error()


@pytest.mark.parametrize("kw,text", [
    (dict(rows=-1), "rows"), (dict(rows=1 << 41), "rows"), (dict(width=0), "width"), (dict(width=1 << 25), "width"), (dict(type=2), "type"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(eps=1e-60), "eps"), (dict(eps=float("inf")), "eps"), (dict(x=None), "x is NULL"), (dict(y=None), "y is NULL"), (dict(ldx=15), "row length of x"),
    (dict(ldy=15), "row length of y"), (dict(x=MB + 1), "not aligned"), (dict(weight=2 * MB + 1), "weight"), (dict(bias=3 * MB + 1), "bias"), (dict(mean=5 * MB + 2), "mean is not aligned"),
    (dict(rstd=6 * MB + 2), "rstd is not aligned"), (dict(y=1 * MB + 2), "y and x" + SHARE), (dict(y=1 * MB, ldy=17), "y and x" + SHARE), (dict(y=2 * MB), "y and weight" + SHARE), (dict(y=3 * MB + 30), "y and bias" + SHARE),
    (dict(mean=1 * MB), "mean and x" + SHARE), (dict(rstd=2 * MB), "rstd and weight" + SHARE), (dict(mean=4 * MB), "y and mean" + SHARE), (dict(rstd=4 * MB + 316), "y and rstd" + SHARE), (dict(rstd=5 * MB + 36), "mean and rstd" + SHARE)])
def test_layer_norm_forward(kw, text):
    refused("cada_layer_norm_forward", cada_norm, NORM, kw, -1, text)


@pytest.mark.parametrize("kw,code,text", [
    (dict(rows=-1), -1, "rows"), (dict(width=0), -1, "width"), (dict(type=3), -1, "type"), (dict(dy=None), -1, "dy is NULL"), (dict(x=None), -1, "x is NULL"), (dict(mean=None), -1, "mean is NULL"), (dict(rstd=None), -1, "rstd is NULL"),
    (dict(lddy=3), -1, "row length of dy"), (dict(ldx=3), -1, "row length of x"), (dict(ldr=3), -1, "row length of residual"), (dict(lddx=3), -1, "row length of dx"), (dict(dw=8 * MB + 1), -1, "dw is not aligned"),
    (dict(db=9 * MB + 1), -1, "db is not aligned"), (dict(weight=5 * MB + 1), -1, "weight"), (dict(workspace=None), -2, "NULL"), (dict(workspace=10 * MB + 16), -2, "256-byte"), (dict(workspace_bytes=100), -2, "too small"),
    (dict(dx=2 * MB), -1, "dx and x" + SHARE), (dict(dx=1 * MB + 2), -1, "dx and dy" + SHARE), (dict(dx=1 * MB, lddx=17), -1, "dx and dy" + SHARE), (dict(dx=6 * MB, lddx=17), -1, "dx and residual" + SHARE),
    (dict(dx=3 * MB), -1, "dx and mean" + SHARE), (dict(dw=1 * MB), -1, "dw and dy" + SHARE), (dict(dw=5 * MB), -1, "dw and weight" + SHARE), (dict(db=8 * MB), -1, "db and dw" + SHARE), (dict(db=7 * MB), -1, "db and dx" + SHARE),
    (dict(workspace=7 * MB), -1, "workspace and dx" + SHARE), (dict(workspace=4 * MB), -1, "workspace and rstd" + SHARE), (dict(workspace=8 * MB), -1, "workspace and dw" + SHARE)])
def test_layer_norm_backward(kw, code, text):
    refused("cada_layer_norm_backward", cada_norm_grad, NORM_GRAD, kw, code, text)


@pytest.mark.parametrize("at", ["dy", "residual"])
def test_dx_in_place_is_not_what_is_refused(at):
    refused("cada_layer_norm_backward", cada_norm_grad, NORM_GRAD, dict(dx=NORM_GRAD[at], dw=5 * MB), -1, "dw and weight" + SHARE)
    refused("cada_layer_norm_backward", cada_norm_grad, NORM_GRAD, dict(rows=1, dx=NORM_GRAD[at], lddx=20, dw=5 * MB), -1, "dw and weight" + SHARE)


def test_y_in_place_is_not_what_is_refused():
    refused("cada_layer_norm_forward", cada_norm, NORM, dict(y=1 * MB, rstd=5 * MB), -1, "mean and rstd" + SHARE)


@pytest.mark.parametrize("name", ["weight", "bias"])
def test_y_in_the_place_of_x_is_not_in_that_of_weights_there(name):
    # (mean and rstd share memory too, so that a call that got past the weights would still be refused before it reached a device)
    refused("cada_layer_norm_forward", cada_norm, NORM, {"y": 1 * MB, name: 1 * MB, "rstd": 5 * MB}, -1, f"y and {name}" + SHARE)


@pytest.mark.parametrize("kw,text", [
    (dict(rows=-1), "rows"), (dict(rows=(1 << 30) + 1), "rows"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 24) + 1), "vocab"), (dict(width=0), "width"), (dict(type=7), "type"), (dict(token_bytes=2), "token_bytes"),
    (dict(scale=float("nan")), "scale"), (dict(scale=1e39), "scale"), (dict(tokens=None), "tokens is NULL"), (dict(tokens=MB + 4), "tokens is not aligned"), (dict(w=None), "w is NULL"), (dict(y=None), "y is NULL"),
    (dict(ldw=3), "row length of w"), (dict(ldy=3), "row length of y"), (dict(w=2 * MB + 1), "w is not aligned"), (dict(y=2 * MB + 99 * 32), "y and w" + SHARE), (dict(y=MB + 72), "y and tokens" + SHARE)])
def test_embedding_forward(kw, text):
    refused("cada_embedding_forward", cada_embedding, EMBED, kw, -1, text)


@pytest.mark.parametrize("kw,code,text", [
    (dict(rows=-1), -1, "rows"), (dict(vocab=0), -1, "vocab"), (dict(vocab=(1 << 24) + 1), -1, "vocab"), (dict(width=0), -1, "width"), (dict(type=2), -1, "type"), (dict(token_bytes=1), -1, "token_bytes"), (dict(scale=float("inf")), -1, "scale"),
    (dict(tokens=None), -1, "tokens is NULL"), (dict(tokens=MB + 2), -1, "tokens is not aligned"), (dict(dy=None), -1, "dy is NULL"), (dict(lddy=15), -1, "row length of dy"), (dict(dw=None), -1, "dw is NULL"), (dict(rows=0, dw=None), -1, "dw is NULL"),
    (dict(lddw=15), -1, "row length of dw"), (dict(workspace=None), -2, "NULL"), (dict(workspace_bytes=1000), -2, "too small"), (dict(dw=2 * MB), -1, "dw and dy" + SHARE), (dict(dw=MB + 3996), -1, "dw and tokens" + SHARE),
    (dict(workspace=2 * MB), -1, "workspace and dy" + SHARE), (dict(workspace=3 * MB), -1, "workspace and dw" + SHARE), (dict(workspace=1 * MB), -1, " and tokens" + SHARE)])
def test_embedding_backward(kw, code, text):
    refused("cada_embedding_backward", cada_embedding_grad, EMBED_GRAD, kw, code, text)


def test_null_arguments_and_sizes():
    for name in ("cada_layer_norm_forward", "cada_layer_norm_backward", "cada_layer_norm_backward_workspace", "cada_embedding_forward", "cada_embedding_backward", "cada_embedding_backward_workspace"):
        assert getattr(_lib, name)(None) == -1 and "NULL" in cada_last_error()
    a = filled(cada_norm_grad, NORM_GRAD, rows=1)
    assert _lib.cada_layer_norm_backward_workspace(C.byref(a)) == 0 and a.workspace_bytes == 0
    a = filled(cada_norm_grad, NORM_GRAD)
    assert _lib.cada_layer_norm_backward_workspace(C.byref(a)) == 0 and a.workspace_bytes >= 2 * 16 * 4
    a = filled(cada_norm_grad, NORM_GRAD, dw=None, db=None)
    assert _lib.cada_layer_norm_backward_workspace(C.byref(a)) == 0 and a.workspace_bytes == 0
    a = filled(cada_embedding_grad, EMBED_GRAD)
    assert _lib.cada_embedding_backward_workspace(C.byref(a)) == 0 and a.workspace_bytes >= 1000 * 8
    a = filled(cada_embedding_grad, EMBED_GRAD, rows=0)
    assert _lib.cada_embedding_backward_workspace(C.byref(a)) == 0 and a.workspace_bytes == 0
    for call, kind, base in (("cada_layer_norm_forward", cada_norm, NORM), ("cada_embedding_forward", cada_embedding, EMBED)):
        assert getattr(_lib, call)(C.byref(filled(kind, base, rows=0, x=None, w=None, y=None) if kind is cada_norm else filled(kind, base, rows=0, tokens=None, y=None))) == 0          # nothing to do


@pytest.mark.parametrize("call", [
    lambda x, v, t: ops.layer_norm_forward(x), lambda x, v, t: ops.layer_norm_backward(x, x, v, v), lambda x, v, t: ops.embedding_forward(t, x), lambda x, v, t: ops.embedding_backward(x, t, 5)])
def test_tensors_that_are_not_on_a_gpu(call):
    with pytest.raises(ValueError, match="GPU"):
        call(torch.zeros(4, 4), torch.zeros(4), torch.zeros(4, dtype=torch.int64))


@pytest.mark.parametrize("call,text", [(lambda: ops.layer_norm_forward(None), "x must be a tensor"), (lambda: ops.embedding_forward(None, None), "tokens must be a tensor"), (lambda: ops.embedding_backward([1.0], None, 4), "dy must be a tensor")])
def test_what_is_no_tensor(call, text):
    with pytest.raises(ValueError, match=text):
        call()


def test_a_residual_that_is_not_needed_is_not_looked_at():
    """Without dx: neither its row length nor where it lies."""
    refused("cada_layer_norm_backward", cada_norm_grad, NORM_GRAD, dict(dx=None, residual=8 * MB, ldr=1, db=8 * MB), -1, "db and dw" + SHARE)
