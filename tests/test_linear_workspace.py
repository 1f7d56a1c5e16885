"""What a layer's calls lay out in their workspaces, by size, on the host: which way operands are read that tiles cannot meet where they lie."""
import ctypes as C

import pytest

from common_ops import cada_linear, cada_linear_grad
from paper_2012_15469_amd.binding import _lib

FAKE = 1 << 20          # an aligned address that nobody reads
F32, BF16 = 0, 1
ELEM = {F32: 4, BF16: 2}


def backward_bytes(rows, k, n, dtype, *, dx=True, dw=True, db=True, act=0, ldw=None):
    a = cada_linear_grad()
    a.rows, a.in_, a.out, a.type, a.act = rows, k, n, dtype, act
    a.dy, a.lddy, a.x, a.ldx, a.w, a.ldw, a.pre, a.ldpre = FAKE, n, FAKE, k, FAKE, ldw or n, FAKE, n
    a.dx, a.lddx, a.dw, a.lddw, a.db = FAKE if dx else None, k, FAKE if dw else None, n, FAKE if db else None
    assert _lib.cada_linear_backward_workspace(C.byref(a)) == 0
    return a.workspace_bytes


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dx_and_db_of_weights_that_tiles_cannot_read(dtype):
    """Below 16 bytes, or rows 2^26 bytes apart: dx is formed element by element from dy itself, and only the parts of db (one per 512 rows) lie in the workspace, no dz for tiles."""
    rows = 200000
    for k, n, ldw in ((1, 1, 1), (1, 3, 3), (3, 1, 1), (40, 5, (1 << 26) // ELEM[dtype])):
        parts = (rows // 512 + 1) * n * 4
        assert parts <= backward_bytes(rows, k, n, dtype, dw=False, ldw=ldw) <= parts + 256 < rows * 8 * ELEM[dtype]
    assert backward_bytes(rows, 40, 5, dtype, dw=False) >= rows * 8 * ELEM[dtype]          # (others by tiles of dz)
