"""Operands and outputs that lie in one another's memory, by addresses that nobody reads: what is refused, and what is not (such a call carries another fault, which is then the one named)."""
import ctypes as C

import pytest

from common_ops import cada_linear
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
