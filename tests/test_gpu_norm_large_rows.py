"""Layer norm's gradients of rows whose mean times rstd passes float32, where (x - mean) rstd is nothing of the sort: lanes without a column hold zeros, whose
distance from such a mean is infinite, and must add nothing to their row's sums.

A constant row has u = (x - mean) rstd = 0 in every column, so dx = rstd (g - mean of g) + residual, and the row's dy enters db but not dw."""
import pytest
import torch

from paper_2012_15469_amd import ops
from test_gpu_norm import DT, check_backward, check_forward, table

pytestmark = pytest.mark.gpu
# a width of every number of lanes and pieces that the gradient has for float32 and bf16, with and without columns behind the last whole piece
WIDTHS = [1, 3, 8, 13, 16, 40, 64, 100, 250, 500, 617, 1000, 1024, 2047, 2048, 4096, 4099, 8190, 9001, 12288, 16381, 16384, 17001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_a_constant_row(width, dtype):
    gen = torch.Generator(device="cuda"); gen.manual_seed(width)
    rows = 7
    x, dy, res, w = table(gen, rows, width, dtype), table(gen, rows, width, dtype), table(gen, rows, width, dtype), table(gen, 1, width, dtype)[0]
    mean, rstd = x.float().mean(1), 1 / torch.sqrt(x.float().var(1, correction=0) + 1e-5)
    # (powers of two: x - mean is exactly zero; 2^121 times 1024 and -2^126 times 32 pass 2^128)
    for row, value, r in ((1, 2.0 ** 121, 1024.0), (4, -2.0 ** 126, 32.0)):
        x[row], mean[row], rstd[row] = value, value, r
    for weight, residual in ((w, res), (None, None), (w, None)):
        check_backward(dy, x, mean, rstd, weight, residual)
        dx = ops.layer_norm_backward(dy, x, mean, rstd, weight, residual=residual, need_dw=False, need_db=False)[0]
        assert bool(torch.isfinite(dx).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [4, 64, 100])
def test_forward_and_backward_of_one(width, dtype):
    """With the default eps, rstd is 316: the same row through both passes."""
    x = torch.full((3, width), 2.0 ** 120, dtype=DT[dtype], device="cuda")
    x[1] = torch.randn(width, device="cuda")
    if width != 100:          # (the mean of 100 such values is not exact in float32)
        _, mean, rstd = check_forward(x[[0, 2]], None, None, 1e-5)
        assert bool((mean == 2.0 ** 120).all())
    y, mean, rstd = ops.layer_norm_forward(x, keep_stats=True)
    dy = torch.randn(3, width, device="cuda").to(x.dtype)
    if width != 100:
        check_backward(dy, x, mean, rstd, None, None)
    assert bool(torch.isfinite(ops.layer_norm_backward(dy, x, mean, rstd)[0][1]).all())
