"""Invalid arguments of a last layer's loss are refused on the host, before anything touches a device; memory that is shared, by addresses that nobody reads."""
import ctypes as C

import pytest

from common_more_ops import cada_linear_xent, filled
from paper_2012_15469_amd.binding import _lib, cada_last_error

MB = 1 << 20
BASE = dict(rows=10, in_=16, classes=40, type=1, label_bytes=8, x=1 * MB, ldx=16, w=2 * MB, ldw=40, bias=3 * MB, labels=4 * MB, ignore_index=-100, smoothing=0.1, scale=1.0, mean=5 * MB, loss=6 * MB,
            dx=7 * MB, lddx=16, dw=8 * MB, lddw=40, db=9 * MB, workspace=10 * MB, workspace_bytes=1 << 28)
SHARE = " share memory"


@pytest.mark.parametrize("kw,code,text", [
    (dict(rows=-1), -1, "rows"), (dict(rows=(1 << 30) + 1), -1, "rows"), (dict(in_=0), -1, "in and classes"), (dict(classes=0), -1, "in and classes"), (dict(classes=1 << 25), -1, "in and classes"), (dict(type=2), -1, "type"),
    (dict(label_bytes=1), -1, "label_bytes"), (dict(smoothing=1.0), -1, "smoothing"), (dict(smoothing=-0.1), -1, "smoothing"), (dict(smoothing=float("nan")), -1, "smoothing"), (dict(rows=1 << 30, classes=1 << 24), -1, "tiles"),
    (dict(x=None), -1, "x is NULL"), (dict(w=None), -1, "w is NULL"), (dict(labels=None), -1, "labels is NULL"), (dict(ldx=15), -1, "row length of x"), (dict(ldw=39), -1, "row length of w"), (dict(lddx=15), -1, "row length of dx"),
    (dict(lddw=39), -1, "row length of dw"), (dict(x=MB + 1), -1, "x is not aligned"), (dict(labels=4 * MB + 4), -1, "labels is not aligned"), (dict(bias=3 * MB + 1), -1, "bias is not aligned"), (dict(db=9 * MB + 1), -1, "db is not aligned"),
    (dict(mean=5 * MB + 2), -1, "mean is not aligned"), (dict(loss=6 * MB + 2), -1, "loss is not aligned"), (dict(workspace=None), -2, "NULL"), (dict(workspace=10 * MB + 64), -2, "256-byte"), (dict(workspace_bytes=4096), -2, "too small"),
    (dict(dx=1 * MB), -1, "dx and x" + SHARE), (dict(dw=2 * MB), -1, "dw and w" + SHARE), (dict(db=3 * MB), -1, "db and bias" + SHARE), (dict(loss=4 * MB), -1, "loss and labels" + SHARE), (dict(mean=4 * MB + 76), -1, "mean and labels" + SHARE),
    (dict(dw=7 * MB), -1, "dw and dx" + SHARE), (dict(db=8 * MB), -1, "db and dw" + SHARE), (dict(mean=6 * MB + 36), -1, "mean and loss" + SHARE), (dict(workspace=7 * MB), -1, "workspace and dx" + SHARE),
    (dict(workspace=1 * MB), -1, "workspace and " ), (dict(loss=1 * MB), -1, "loss and x" + SHARE)])
def test_refused(kw, code, text):
    assert _lib.cada_linear_cross_entropy(C.byref(filled(cada_linear_xent, BASE, **kw))) == code and text in cada_last_error(), cada_last_error()


def size(**kw):
    a = filled(cada_linear_xent, BASE, **kw)
    assert _lib.cada_linear_xent_workspace(C.byref(a)) == 0
    return a.workspace_bytes


def test_sizes():
    assert _lib.cada_linear_xent_workspace(None) == -1 and _lib.cada_linear_cross_entropy(None) == -1
    assert size(rows=0) == 0
    none = dict(dx=None, dw=None, db=None)
    assert size(**none) < size(dx=None, dw=None) < size()
    big = dict(rows=8192, in_=1024, ldx=1024, classes=65536, ldw=65536, lddx=1024, lddw=65536, smoothing=0.0)
    logits = 8192 * 65536 * 2
    assert size(**big, **none) < logits / 12 and size(**big) < logits / 2          # without the logits
    # many rows: a statistic of 8 bytes for every 64 logits, x and its gradient in float32, a piece's signal, and parts of a piece's dw
    assert size(**{**big, "rows": 131072}) < 16 * logits * 8 / 128 + 131072 * 1024 * (2 + 4) + 131072 * 1024 * 2 + (1 << 27)
