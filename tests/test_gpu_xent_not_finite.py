"""Rows of logits that hold NaN or infinities, in every group of lanes that a row can have: NaN and +inf show in the loss, its mean and the gradient whatever else is in the row, and only a row
with every class ruled out counts as one with nothing left."""
import math

import pytest
import torch

from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("n", [1, 2, 3, 7, 30, 60, 100, 200, 500, 1001, 2500, 7000, 14000, 20011, 50001, 100003, 140001])
def test_not_a_number_shows(n, dtype):
    for smoothing in (0.0, 0.1):
        for place in sorted({0, n // 2, n - 1}):
            z = torch.randn(9, n, device="cuda").to(dtype)
            labels = torch.arange(9, device="cuda") % n
            z[1] = NAN
            z[2] = -INF; z[2, place] = NAN
            z[3, place] = NAN
            z[4, place] = INF
            z[5] = -INF
            z[6] = NAN
            labels[6] = -100                     # (ignored: nothing in it counts)
            z[7] = -INF; z[7, place] = 1.0
            labels[7] = place
            mean, loss, grad = ops.cross_entropy(z, labels, smoothing=smoothing)
            for row in (1, 2, 3, 4):
                assert torch.isnan(loss[row]) and torch.isnan(grad[row, place]), (row, smoothing, place)
            assert torch.isnan(grad[1]).all() and torch.isnan(grad[2]).all() and torch.isnan(grad[3]).all()
            assert loss[5] == INF and not grad[5].float().any()
            assert float(loss[6]) == 0.0 and not grad[6].float().any()
            assert float(loss[7]) == 0.0 and not grad[7].float().any()
            assert torch.isfinite(loss[[0, 8]]).all() and torch.isfinite(grad[[0, 8]]).all() and torch.isnan(mean)
            # by itself (rows of one workgroup are counted there)
            for row in (1, 2):
                mean, loss, grad = ops.cross_entropy(z[row:row + 1], labels[row:row + 1], smoothing=smoothing)
                assert torch.isnan(mean) and torch.isnan(loss[0]) and torch.isnan(grad).all()
            mean, loss, grad = ops.cross_entropy(z[5:6], labels[5:6], smoothing=smoothing)
            assert float(mean) == INF and float(loss[0]) == INF and not grad.float().any()
