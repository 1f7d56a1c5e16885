"""Layer norm of more rows than a launch has groups of lanes (2048 workgroups forward, 1024 of 512 lanes; 512 and 256 backward; up to 64 rows of a workgroup at
once): a group takes several rows, the next of which is asked for before a row is written, also where it is written in the place of what was read, and the
last turn is partly filled."""
import pytest
import torch

from paper_2012_15469_amd import ops
from test_gpu_norm import check_backward, check_forward, table

pytestmark = pytest.mark.gpu
# two turns or three forward, of each number of lanes and pieces of float32 or bf16 rows (the last: past the registers of float32), and up to seventeen backward
MANY = [(140003, 13), (70001, 40), (40003, 100), (17001, 250), (16389, 500), (8203, 1001), (8199, 2047), (2049, 4096), (2051, 8190), (1027, 9001), (1030, 16383), (1026, 32761), (2400, 617)]
WIDE = 4


def in_wider(t, fill=7.0):
    """A copy of t's values in rows of a wider table, and the columns behind them."""
    wide = torch.full((t.shape[0], t.shape[1] + WIDE), fill, dtype=t.dtype, device="cuda")
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]], wide[:, t.shape[1]:]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", MANY)
def test_turns(rows, width, dtype):
    gen = torch.Generator(device="cuda"); gen.manual_seed(rows + width)
    x, w, b = table(gen, rows, width, dtype, 3, 1, 2.0, 0.3), table(gen, 1, width, dtype, place=1.0)[0], table(gen, 1, width, dtype)[0]
    y, m, r = check_forward(x, w, b, 1e-5)
    z, behind = in_wider(x)
    again = ops.layer_norm_forward(z, w, b, keep_stats=True, out=z)
    assert all(torch.equal(a, c) for a, c in zip(again, (y, m, r))) and bool((behind == 7.0).all())
    del again, z, behind
    dy, res = table(gen, rows, width, dtype, 5), table(gen, rows, width, dtype)
    first = check_backward(dy, x, m, r, w, res)
    for place in ("dy", "residual"):
        a, c = in_wider(dy), in_wider(res)
        out, behind = a if place == "dy" else c
        got = ops.layer_norm_backward(a[0], x, m, r, w, residual=c[0], dx=out)
        assert got[0] is out and all(torch.equal(g, f) for g, f in zip(got, first)) and bool((behind == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", [(8199, 617), (2051, 4096), (1030, 9001)])
def test_no_turn_sees_another(rows, width, dtype):
    """A row of NaN, infinities or the largest values changes its own results only, whichever turn it comes in (but for the sums over the rows, which are not
    asked for)."""
    gen = torch.Generator(device="cuda"); gen.manual_seed(width)
    x, dy, w = table(gen, rows, width, dtype), table(gen, rows, width, dtype), table(gen, 1, width, dtype)[0]
    y, m, r = ops.layer_norm_forward(x, w, keep_stats=True)
    dx = ops.layer_norm_backward(dy, x, m, r, w, need_dw=False, need_db=False)[0]
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[::37] = True
    bad[-1] = True
    x2, dy2 = x.clone(), dy.clone()
    x2[bad, 0] = float("nan")
    dy2[bad, width - 1] = float("inf")
    y2, m2, r2 = ops.layer_norm_forward(x2, w, keep_stats=True, out=x2.clone())
    assert torch.equal(y2[~bad], y[~bad]) and torch.equal(m2[~bad], m[~bad]) and torch.equal(r2[~bad], r[~bad]) and bool(torch.isnan(y2[bad]).all())
    dx2 = ops.layer_norm_backward(dy2, x, m, r, w, need_dw=False, need_db=False)[0]
    assert torch.equal(dx2[~bad], dx[~bad]) and not bool(torch.isfinite(dx2[bad]).all(1).any())
