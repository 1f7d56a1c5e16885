"""Which tiles a layer's products take (csrc/cada_linear_plan.h), on the host: the offsets of a tile's pieces, which the kernels hold in 32 bits, do not wrap."""
import ctypes as C
import os
import random
import subprocess

import pytest

from common_ops import cada_linear, cada_linear_grad

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20          # an aligned address that nobody reads
ELEM = {0: 4, 1: 2}

_SRC = """
#include "cada_linear_plan.h"
using namespace cada;
extern "C" {
void forward(const cada_linear *a, long *out) {
  const ForwardPlan f = plan_forward(a);
  const long v[] = {f.few, f.by_element, f.direct, f.pack_x, f.pack_w, f.cut.tile};
  std::copy(v, v + 6, out);
}
void backward(const cada_linear_grad *a, long *out) {
  const BackwardPlan b = plan_backward(a);
  const long v[] = {b.small, b.by_element, b.own_dz, b.direct, b.pack_x, b.pack_w, b.dx.tile, b.dw.tile, (long)b.lddz};
  std::copy(v, v + 9, out);
}
long packed(long cols) { return packed_ld(cols); }
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
    return dll


def forward(plan, rows, k, n, dtype, ldx=None, ldw=None, shift=0):
    a = cada_linear()
    a.rows, a.in_, a.out, a.type, a.act = rows, k, n, dtype, 0
    a.x, a.ldx, a.w, a.ldw = FAKE + shift, ldx or k, FAKE + shift, ldw or n
    v = (C.c_long * 6)()
    plan.forward(C.byref(a), v)
    return dict(zip(("few", "by_element", "direct", "pack_x", "pack_w", "tile"), v)), a


def backward(plan, rows, k, n, dtype, act=0, dx=True, dw=True, db=True, ldx=None, ldw=None, lddy=None, shift=0):
    a = cada_linear_grad()
    a.rows, a.in_, a.out, a.type, a.act = rows, k, n, dtype, act
    a.dy, a.lddy, a.x, a.ldx, a.w, a.ldw, a.pre, a.ldpre = FAKE + shift, lddy or n, FAKE + shift, ldx or k, FAKE + shift, ldw or n, FAKE, n
    a.dx, a.lddx, a.dw, a.lddw, a.db = FAKE if dx else None, k, FAKE if dw else None, n, FAKE if db else None
    v = (C.c_long * 9)()
    plan.backward(C.byref(a), v)
    return dict(zip(("small", "by_element", "own_dz", "direct", "pack_x", "pack_w", "tile_dx", "tile_dw", "lddz"), v)), a


def furthest(ld, along, tile, elem):
    """Offset of the last byte of a tile's pieces: a tile's rows of a step's 128 bytes (along the contraction), or a step's rows of a tile's columns."""
    return ((tile - 1) * ld * elem + 128) if along else (128 // elem - 1) * ld * elem + tile * elem


def check_forward(plan, *args, **kw):
    p, a = forward(plan, *args, **kw)
    if p["few"] or p["by_element"]:
        return
    ldx = plan.packed(a.in_) if p["pack_x"] else a.ldx
    ldw = plan.packed(a.out) if p["pack_w"] else a.ldw
    assert furthest(ldx, True, p["tile"], ELEM[a.type]) < 1 << 32 and furthest(ldw, False, p["tile"], ELEM[a.type]) < 1 << 32, (args, kw, p)


def check_backward(plan, *args, **kw):
    p, a = backward(plan, *args, **kw)
    if p["by_element"]:
        return
    lddz = p["lddz"] if p["own_dz"] else a.lddy
    elem = ELEM[a.type]
    if a.dx:
        ldw = plan.packed(a.out) if p["pack_w"] else a.ldw
        assert furthest(lddz, True, p["tile_dx"], elem) < 1 << 32 and furthest(ldw, True, p["tile_dx"], elem) < 1 << 32, (args, kw, p)
    if a.dw:
        ldx = plan.packed(a.in_) if p["pack_x"] else a.ldx
        assert furthest(ldx, False, p["tile_dw"], elem) < 1 << 32 and furthest(lddz, False, p["tile_dw"], elem) < 1 << 32, (args, kw, p)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("long", [(1 << 22) + 64, (1 << 23) - 4, 1 << 23, (1 << 23) + 64, (1 << 24) - 8, (1 << 24) - 1, 1 << 24])
def test_offsets_of_long_contractions(plan, long, dtype):
    for rows in (3, 130, 256, 300, 1024, 4096):
        for other in (8, 40, 256, 1000, 1024, 4096):
            for shift in (0, ELEM[dtype]):
                check_forward(plan, rows, long, other, dtype, shift=shift)
                check_forward(plan, rows, other, long, dtype, shift=shift)
                for need in ((True, True), (True, False), (False, True)):
                    for act in (0, 2):
                        if max(-(-rows // 64), -(-other // 64)) * (-(-long // 64)) < 1 << 23:
                            check_backward(plan, rows, other, long, dtype, act, *need, shift=shift)
                            check_backward(plan, rows, long, other, dtype, act, *need, shift=shift)


def test_offsets_of_rows_far_apart(plan):
    rng = random.Random(1)
    for _ in range(20000):
        dtype = rng.choice((0, 1))
        rows, k, n = (int(2 ** rng.uniform(0, 13)) for _ in range(3))
        lds = [max(w, int(2 ** rng.uniform(3, 28)) // 8 * 8 + rng.choice((0, 0, 3))) for w in (k, n, n)]
        check_forward(plan, rows, k, n, dtype, ldx=lds[0], ldw=lds[1])
        check_backward(plan, rows, k, n, dtype, rng.choice((0, 1)), rng.random() < 0.7, rng.random() < 0.7, rng.random() < 0.5, ldx=lds[0], ldw=lds[1], lddy=lds[2])


def test_every_table_that_tiles_read_holds_a_piece(plan):
    """A load through registers takes 16 bytes and is moved back from a table's end so as to lie in it: tables of less are read element by element."""
    rng = random.Random(2)
    spans = lambda rows, ld, cols, elem: ((rows - 1) * ld + cols) * elem
    for _ in range(100000):
        dtype = rng.choice((0, 1))
        rows, k, n = (rng.choice((1, 1, 2, 3, rng.randint(1, 9), int(2 ** rng.uniform(0, 12)))) for _ in range(3))
        pad, shift = [rng.choice((0, 0, 1, 8)) for _ in range(3)], rng.choice((0, ELEM[dtype]))
        lds = [w + p for w, p in zip((k, n, n), pad)]
        elem = ELEM[dtype]
        p, a = forward(plan, rows, k, n, dtype, ldx=lds[0], ldw=lds[1], shift=shift)
        if not p["few"] and not p["by_element"]:
            assert spans(rows, plan.packed(k) if p["pack_x"] else lds[0], k, elem) >= 16 and spans(k, plan.packed(n) if p["pack_w"] else lds[1], n, elem) >= 16
        dx, dw, db = (rng.random() < 0.6 for _ in range(3))
        p, a = backward(plan, rows, k, n, dtype, rng.choice((0, 1)), dx, dw, db, ldx=lds[0], ldw=lds[1], lddy=lds[2], shift=shift)
        if (dx or dw) and not p["by_element"]:
            what = (rows, k, n, dtype, dx, dw, db, lds, p)
            assert spans(rows, p["lddz"] if p["own_dz"] else lds[2], n, elem) >= 16, what
            assert not p["small"] or a.act == 0 or spans(rows, n, n, elem) >= 16, what          # (pre)
            assert not dx or spans(k, plan.packed(n) if p["pack_w"] else lds[1], n, elem) >= 16, what
            assert not dw or spans(rows, plan.packed(k) if p["pack_x"] else lds[0], k, elem) >= 16, what
