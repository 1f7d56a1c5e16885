"""dx and db without dw: the weights that this reads may be smaller than a read of 16 bytes, or their rows too far apart for a tile's offsets."""
import pytest
import torch

from paper_2012_15469_amd import ops
from test_gpu_linear_integers import DT, ints, rounded

pytestmark = pytest.mark.gpu


def gradients(dy, x, w, pre, act, dtype):
    dx, dw, db = ops.linear_backward(dy, x, w, pre=pre, act=act, need_dw=False)
    dz = dy.double() * ((pre.double() > 0).double() if pre is not None else 1.0)
    assert dw is None and torch.equal(dx, rounded(dz @ w.double().t(), dtype)) and torch.equal(db, rounded(dz.sum(0), dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,n", [(1, 1), (1, 2), (1, 3), (2, 1), (3, 1), (2, 2), (2, 3), (3, 2), (7, 1), (1, 7), (4, 1), (1, 4), (1, 8), (8, 1), (5, 3), (40, 1), (1, 40), (33, 70)], ids=str)
def test_small_weights(k, n, dtype):
    gen = torch.Generator(device="cuda"); gen.manual_seed(k * 50 + n)
    for rows in (1, 2, 5, 70, 1000, 20003):
        for pad in (0, 3):
            for act in ("none", "relu"):
                # (weights in the middle of a larger tensor of NaN: nothing around them matters)
                around = torch.full((64 + k * (n + pad),), float("nan"), device="cuda", dtype=DT[dtype])
                w = around[33:33 + k * (n + pad)].view(k, n + pad)[:, :n]
                w.copy_(ints(k, n, dtype, gen))
                dy, x = ints(rows, n, dtype, gen, pad), ints(rows, k, dtype, gen, pad)
                gradients(dy, x, w, ints(rows, n, dtype, gen) if act == "relu" else None, act, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_rows_far_apart(dtype):
    k, n, rows = 40, 5, 70
    ld = (1 << 26) // (2 if dtype == "bf16" else 4)          # 64 rows are 2^32 bytes apart
    gen = torch.Generator(device="cuda"); gen.manual_seed(2)
    w = torch.empty((k - 1) * ld + n, dtype=DT[dtype], device="cuda").as_strided((k, n), (ld, 1))
    w.copy_(ints(k, n, dtype, gen))
    for act in ("none", "relu"):
        gradients(ints(rows, n, dtype, gen), ints(rows, k, dtype, gen), w, ints(rows, n, dtype, gen) if act == "relu" else None, act, dtype)
