"""How the loss of a last layer's product is cut (csrc/cada_linear_plan.h), on the host: its pieces cover the classes, its parts of the workspace lie one behind the other, offsets of a tile's pieces, which the kernels hold in 32 bits, do not wrap."""
import ctypes as C
import os
import random
import subprocess

import pytest

from common_more_ops import cada_linear_xent, filled

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20          # an aligned address that nobody reads
ELEM = {0: 4, 1: 2}
NAMES = ("grads", "signal", "kept", "left", "wide", "direct", "copy_x", "copy_w", "outer", "tile", "splits", "piece_tile", "dx_tile", "dx_splits", "dx_per", "dw_tile", "dw_splits", "dw_per", "piece", "pieces", "chunks", "ldz", "strips", "left_rows", "floats",
         "bias", "stats", "left_at", "info", "label", "loss", "signal_at", "dx", "dw", "db", "x", "w", "bytes")
_SRC = """
#include "cada_linear_plan.h"
using namespace cada;
extern "C" {
void plan(const cada_linear_xent *a, long *out) {
  const LossPlan f = plan_loss(a);
  const long v[] = {f.grads, f.signal, f.kept, f.left, f.wide, f.direct, f.copy_x, f.copy_w, f.outer, f.logits.tile, f.logits.splits, f.piece_logits.tile, f.dx.tile, f.dx.splits, (long)f.dx.k_per_split, f.dw.tile, f.dw.splits, (long)f.dw.k_per_split,
                    (long)f.piece, (long)f.pieces, (long)f.chunks, (long)f.ldz, (long)f.strips, (long)f.left_rows, f.stat_floats, (long)f.off_bias, (long)f.off_stats, (long)f.off_left, (long)f.off_info, (long)f.off_label, (long)f.off_loss, (long)f.off_signal,
                    (long)f.off_dx, (long)f.off_dw, (long)f.off_db, (long)f.off_x, (long)f.off_w, (long)f.bytes};
  std::copy(v, v + sizeof(v) / sizeof(v[0]), out);
}
long packed(long cols) { return packed_ld(cols); }
long most_groups() { return kMostGroups; }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    tmp = str(tmp_path_factory.mktemp("plan"))
    src, lib = os.path.join(tmp, "plan.cc"), os.path.join(tmp, "plan.so")
    with open(src, "w") as f:
        f.write(_SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2012_15469_amd", "csrc"), "-I", os.path.join(ROOT, "include"), "-o", lib, src], check=True)
    dll = C.CDLL(lib)
    dll.packed.restype, dll.packed.argtypes = C.c_long, [C.c_long]

    def call(rows, k, classes, dtype, ldx=None, ldw=None, shift=0, outs=(1, 1, 1), smoothing=0.0):
        a = filled(cada_linear_xent, dict(rows=rows, in_=k, classes=classes, type=dtype, label_bytes=8, x=FAKE + shift, ldx=ldx or k, w=FAKE + shift, ldw=ldw or classes, labels=FAKE, smoothing=smoothing,
                                          dx=FAKE if outs[0] else None, lddx=k, dw=FAKE if outs[1] else None, lddw=classes, db=FAKE if outs[2] else None))
        v = (C.c_long * len(NAMES))()
        dll.plan(C.byref(a), v)
        return dict(zip(NAMES, v)), a, dll
    return call


def check(f, a, dll):
    rows, k, classes, elem = a.rows, a.in_, a.classes, ELEM[a.type]
    e8 = lambda n: -(-n // 8) * 8  # noqa: E731
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    assert f["pieces"] >= 1 and (f["pieces"] - 1) * f["piece"] < classes <= f["pieces"] * f["piece"] and (f["pieces"] == 1 or f["piece"] % 256 == 0) and f["ldz"] >= f["piece"]
    assert f["tile"] in (32, 64, 128, 256) and (f["direct"] or f["tile"] <= 64) and (a.type == 1 or f["tile"] <= 64)
    if f["kept"]:
        assert f["signal"] and f["pieces"] == 1 and classes <= 16384 and not f["left"] and f["splits"] * rows * e8(classes) * 4 <= 192 << 20 and f["strips"] <= dll.most_groups()
    else:
        assert not f["wide"] or (rows <= 64 and a.type == 1 and f["tile"] == 64 and f["chunks"] == -(-classes // 128) * 4)
        assert f["splits"] == 1 and f["chunks"] * {256: 64}.get(f["tile"], 32) >= classes
        if f["left"]:
            assert f["signal"] and f["pieces"] == 1 and classes > 16384 and rows * e8(classes) * 4 <= 192 << 20 and f["strips"] * f["left_rows"] >= rows and f["strips"] < 65536
        elif f["signal"]:
            assert f["strips"] * f["piece_tile"] // 2 >= rows
    # the workspace
    sizes = [("bias", e8(classes) * 4 if f["kept"] else 0), ("stats", f["splits"] * rows * e8(classes) * 4 if f["kept"] else f["chunks"] * rows * f["floats"] * 4), ("left_at", rows * e8(classes) * 4 if f["left"] else 0), ("info", rows * 16), ("label", rows * 4), ("loss", 0 if a.loss else rows * 4),
             ("signal_at", rows * f["ldz"] * elem if f["grads"] else 0), ("dx", f["dx_splits"] * rows * e8(k) * 4 if a.dx and (f["pieces"] > 1 or f["dx_splits"] > 1) else 0),
             ("dw", f["dw_splits"] * k * e8(f["piece"]) * 4 if a.dw and not f["outer"] and f["dw_splits"] > 1 else 0), ("db", f["strips"] * f["piece"] * 4 if a.db else 0), ("x", rows * dll.packed(k) * elem if f["copy_x"] else 0),
             ("w", k * dll.packed(classes) * elem if f["copy_w"] else 0)]
    ends = [f[name] for name, _ in sizes[1:]] + [f["bytes"]]
    assert f["bias"] >= 1024
    for (name, size), end in zip(sizes, ends):
        assert f[name] + size <= end and f[name] % 256 == 0 and end - f[name] <= up(size), name
    # offsets of a tile's rows, and of the rows of a step of the contraction, in bytes
    ldx, ldw = dll.packed(k) if f["copy_x"] else a.ldx, dll.packed(classes) if f["copy_w"] else a.ldw
    step = 128 // elem
    tiles = [f["tile"]] + ([f["piece_tile"]] if f["signal"] and not f["kept"] else [])
    for tile in tiles:
        assert tile * ldx * elem <= 1 << 32 and step * ldw * elem <= 1 << 32
    if a.dx:
        assert f["dx_tile"] * f["ldz"] * elem <= 1 << 32 and f["dx_tile"] * ldw * elem <= 1 << 32
        assert f["dx_splits"] * f["dx_per"] >= f["piece"] > (f["dx_splits"] - 1) * f["dx_per"]
    assert f["outer"] == (bool(a.dw) and rows <= 16)
    if a.dw and not f["outer"]:
        assert step * ldx * elem <= 1 << 32 and step * f["ldz"] * elem <= 1 << 32
        assert f["dw_splits"] * f["dw_per"] >= rows > (f["dw_splits"] - 1) * f["dw_per"]
    if a.dx and a.dw and not f["outer"]:
        assert f["dx_tile"] == f["dw_tile"]
    # tables that are read directly: rows on 16-byte boundaries, whole pieces
    if f["direct"]:
        assert f["copy_x"] or (a.x % 16 == 0 and a.ldx * elem % 16 == 0)
        assert f["copy_w"] or (a.w % 16 == 0 and a.ldw * elem % 16 == 0 and classes * elem % 16 == 0)
    # tables of less than a load are copied, so that what lies before them is the workspace's
    for rows_, ld, cols, copied in ((rows, a.ldx, k, f["copy_x"]), (k, a.ldw, classes, f["copy_w"])):
        assert ((rows_ - 1) * ld + cols) * elem >= 16 or copied


@pytest.mark.parametrize("dtype", [0, 1])
def test_drawn(plan, dtype):
    rng = random.Random(dtype)
    for _ in range(3000):
        rows, k, classes = (max(1, int(2 ** rng.uniform(0, b))) for b in (18, 13, 18))
        while rows * classes > 1 << 33 or -(-rows // 64) * -(-classes // 64) > 1 << 23:
            rows = max(1, rows // 2)
        if rng.random() < 0.5:
            k, classes = max(8, k // 16 * 16), max(8, classes // 16 * 16)
        pad = rng.choice([0, 0, 8, 3])
        check(*plan(rows, k, classes, dtype, k + pad, classes + pad, rng.choice([0, 0, 0, ELEM[dtype]]), rng.choice([(1, 1, 1), (1, 1, 0), (0, 0, 0), (1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1)]), rng.choice([0.0, 0.1])))


@pytest.mark.parametrize("rows,k,classes,dtype,ldx,ldw", [
    (1, 1, 1, 0, 1, 1), (1, 1, 1, 1, 1, 1), (1, 7, 1, 1, 7, 1), (3, 1, 2, 1, 1, 2), (64, 64, 1 << 24, 1, 64, 1 << 24), (64, 64, 1 << 24, 0, 64, 1 << 24), (64, 1 << 24, 64, 1, 1 << 24, 64), (300, 64, 4096, 1, 1 << 28, 4096),
    (300, 64, 4096, 1, 64, 1 << 28), (300, 65, 4097, 0, 1 << 27, 1 << 27), (8192, 4096, 65536, 1, 4096, 65536), (1 << 20, 64, 50001, 1, 64, 50001)])
def test_extremes(plan, rows, k, classes, dtype, ldx, ldw):
    for outs in ((1, 1, 1), (0, 0, 0), (1, 0, 0), (0, 1, 0)):
        check(*plan(rows, k, classes, dtype, ldx, ldw, 0, outs))
