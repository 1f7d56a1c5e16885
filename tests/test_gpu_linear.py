"""A layer's product and its gradients against the formulas in 64 bits.

Tolerances, elementwise: a sum of k products in float32 is off by at most (k + 8) 2^-23 sum |x||w| (every product and every addition rounds once,
with room for the bias and the activation, whose slope is below 1.2); writing bf16 adds 2^-8 of the value, and in the gradients dz
was rounded to bf16 before the products, 2^-8 of sum |dz||.|."""
import math

import pytest
import torch

from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def act64(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z)}[act]()


def slope64(z, act):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(),
            "gelu": lambda: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), "silu": lambda: s + z * s * (1 - s)}[act]()


def table(rows, cols, dtype, gen, pad=0, shift=0, scale=1.0):
    """A [rows, cols] tensor; `pad` more elements from row to row, the first one `shift` elements into the memory."""
    t = torch.randn(rows, cols + pad + shift, generator=gen, device="cuda") * scale
    return t.to(DT[dtype])[:, shift:shift + cols]


def rounding(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22


def close(got, want, bound, dtype):
    assert got.shape == want.shape
    err = (got.double() - want).abs()
    limit = bound * 1.2 + rounding(dtype) * want.abs() + 1e-30
    worst = float((err / limit).max()) if err.numel() else 0.0
    assert worst <= 1.0, worst


SHAPES = [(1, 1, 1), (1, 64, 64), (1, 1000, 333), (2, 7, 3), (3, 130, 200), (8, 512, 64), (9, 65, 129), (17, 617, 301), (63, 64, 65), (64, 128, 10), (65, 33, 128), (127, 300, 256),
          (130, 784, 500), (200, 1024, 72), (257, 100, 520), (1030, 72, 1000), (520, 2050, 640), (2048, 16, 2048), (4097, 136, 24), (5, 8200, 10), (3000, 40, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype):
    rows, k, n = shape
    gen = torch.Generator(device="cuda"); gen.manual_seed(rows * 7 + k)
    for act, pad, shift, residual, bias in (("none", 0, 0, False, False), ("relu", 8, 0, True, True), ("gelu", 3, 1, True, True), ("silu", 0, 0, False, True)):
        x, w = table(rows, k, dtype, gen, pad, shift), table(k, n, dtype, gen, pad, shift, 1 / math.sqrt(k))
        b = table(1, n, dtype, gen)[0] if bias else None
        r = table(rows, n, dtype, gen, pad, shift) if residual else None
        y, pre = ops.linear_forward(x, w, b, residual=r, act=act, keep_pre=True)
        y2, none = ops.linear_forward(x, w, b, residual=r, act=act)
        assert none is None and torch.equal(y, y2)
        z = x.double() @ w.double() + (b.double() if bias else 0)
        bound = (k + 8) * U * (x.double().abs() @ w.double().abs() + (b.double().abs() if bias else 0))
        close(pre, z, bound, dtype)
        close(y, act64(z, act) + (r.double() if residual else 0), bound + U * (r.double().abs() if residual else 0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype):
    rows, k, n = shape
    gen = torch.Generator(device="cuda"); gen.manual_seed(rows * 11 + n)
    for act, pad, shift in (("none", 0, 0), ("relu", 8, 0), ("gelu", 3, 1), ("silu", 0, 0), ("none", 1, 0)):
        x, w, dy = table(rows, k, dtype, gen, pad, shift), table(k, n, dtype, gen, pad, shift, 1 / math.sqrt(k)), table(rows, n, dtype, gen, pad, shift)
        pre = table(rows, n, dtype, gen, pad, shift) if act != "none" else None
        dx, dw, db = ops.linear_backward(dy, x, w, pre=pre, act=act)
        dz = dy.double() * (slope64(pre.double(), act) if pre is not None else 1)
        dz_abs, r = dy.double().abs() * 1.2, 2.0 ** -8 if dtype == "bf16" and act != "none" else 0.0      # (a slope near zero is off by a few U of its terms, not of itself)
        want = (dz @ w.double().t(), x.double().t() @ dz, dz.sum(0))
        bound = (((n + 16) * U + r) * (dz_abs @ w.double().abs().t()), ((rows + 16) * U + r) * (x.double().abs().t() @ dz_abs), (rows + 16) * U * dz_abs.sum(0))
        for got, v, bd in zip((dx, dw, db), want, bound):
            close(got, v, bd, dtype)
        # each output alone (the contractions may be cut otherwise)
        for need in ((True, False, False), (False, True, False), (False, False, True)):
            alone = ops.linear_backward(dy, x, w, pre=pre, act=act, need_dx=need[0], need_dw=need[1], need_db=need[2])
            for wanted, got, v, bd in zip(need, alone, want, bound):
                if wanted:
                    close(got, v, bd, dtype)
                else:
                    assert got is None


# Large enough for every tile that the library has (bf16; float32 has one), with and without 16-byte rows, and contractions that end inside a step.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(8200, 2056, 4104), (4100, 1032, 1032), (2056, 520, 2056), (3001, 1001, 1003), (300, 4100, 520)], ids=str)
def test_large(shape, dtype):
    rows, k, n = shape
    gen = torch.Generator(device="cuda"); gen.manual_seed(rows)
    x, w, b, r = table(rows, k, dtype, gen), table(k, n, dtype, gen, scale=1 / math.sqrt(k)), table(1, n, dtype, gen)[0], table(rows, n, dtype, gen)
    y, pre = ops.linear_forward(x, w, b, residual=r, act="gelu", keep_pre=True)
    z = x.double() @ w.double() + b.double()
    bound = (k + 8) * U * (x.double().abs() @ w.double().abs() + b.double().abs())
    close(pre, z, bound, dtype)
    close(y, act64(z, "gelu") + r.double(), bound + U * r.double().abs(), dtype)
    dx, dw, db = ops.linear_backward(r, x, w, pre=pre, act="gelu")
    dz, extra = r.double() * slope64(pre.double(), "gelu"), 2.0 ** -8 if dtype == "bf16" else 0.0
    close(dx, dz @ w.double().t(), ((n + 16) * U + extra) * (r.double().abs() @ w.double().abs().t()), dtype)
    close(dw, x.double().t() @ dz, ((rows + 16) * U + extra) * (x.double().abs().t() @ r.double().abs()), dtype)
    close(db, dz.sum(0), (rows + 16) * U * r.double().abs().sum(0) * 1.2, dtype)


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradient_against_differences(act):
    """Central differences of the formula in 64 bits, step 1e-5: their own error is below 1e-8 here; float32 gradients are off by (k + 16) U of their terms, 1e-5."""
    gen = torch.Generator(device="cuda"); gen.manual_seed(5)
    rows, k, n, h = 6, 9, 7, 1e-5
    x, w, b, r = table(rows, k, "f32", gen), table(k, n, "f32", gen), table(1, n, "f32", gen)[0], table(rows, n, "f32", gen)
    dy = table(rows, n, "f32", gen)
    y, pre = ops.linear_forward(x, w, b, residual=r, act=act, keep_pre=True)
    got = ops.linear_backward(dy, x, w, pre=pre, act=act)
    value = lambda x, w, b: float(((act64(x @ w + b, act) + r.double()) * dy.double()).sum())
    args = [x.double(), w.double(), b.double()]
    for i, g in enumerate(got):
        num = torch.zeros_like(args[i])
        for j in range(num.numel()):
            hi, lo = [a.clone() for a in args], [a.clone() for a in args]
            hi[i].view(-1)[j] += h
            lo[i].view(-1)[j] -= h
            num.view(-1)[j] = (value(*hi) - value(*lo)) / (2 * h)
        assert torch.allclose(g.double(), num, rtol=1e-4, atol=1e-4), float((g.double() - num).abs().max())


def test_no_rows():
    for dt in DT.values():
        x, w, b = torch.empty(0, 70, dtype=dt, device="cuda"), torch.randn(70, 33, device="cuda").to(dt), torch.randn(33, device="cuda").to(dt)
        y, pre = ops.linear_forward(x, w, b, act="relu", keep_pre=True)
        assert y.shape == pre.shape == (0, 33)
        dx, dw, db = ops.linear_backward(y, x, w, pre=pre, act="relu", dw=torch.full((70, 33), 7.0, dtype=dt, device="cuda"), db=torch.full((33,), 7.0, dtype=dt, device="cuda"))
        assert dx.shape == (0, 70) and float(dw.float().abs().sum()) == 0.0 and float(db.float().abs().sum()) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 200, 70), (5, 136, 64), (130, 200, 136), (300, 77, 131)], ids=str)
def test_nothing_outside_the_operands_matters(shape, dtype):
    """What lies between and behind the rows is NaN, the outputs' surroundings stay as they are, and infinities and NaN reach only what depends on them."""
    rows, k, n = shape
    gen = torch.Generator(device="cuda"); gen.manual_seed(9)
    for pad in (8, 5):
        def framed(r, c):
            big = torch.full((r + 2, c + pad + 8), math.nan, device="cuda", dtype=DT[dtype])
            inner = big[1:1 + r, 8:8 + c]
            inner.copy_(torch.randn(r, c, generator=gen, device="cuda"))
            return big, inner
        x, w, r, pre, dy = (framed(*s)[1] for s in ((rows, k), (k, n), (rows, n), (rows, n), (rows, n)))
        outs = [framed(*s) for s in ((rows, n), (rows, n), (rows, k), (k, n))]
        before = [big.clone() for big, _ in outs]
        ops.linear_forward(x, w, None, residual=r, act="silu", out=outs[0][1], pre=outs[1][1])
        ops.linear_backward(dy, x, w, pre=pre, act="silu", dx=outs[2][1], dw=outs[3][1])
        for (big, inner), old in zip(outs, before):
            assert torch.isfinite(inner).all()
            now = big.clone()
            now[1:1 + inner.shape[0], 8:8 + inner.shape[1]] = old[1:1 + inner.shape[0], 8:8 + inner.shape[1]]
            assert torch.equal(torch.nan_to_num(now, nan=-3.0), torch.nan_to_num(old, nan=-3.0))
        xi = x.clone()
        xi[0, k - 1] = math.inf
        y, _ = ops.linear_forward(xi, w)
        assert not torch.isfinite(y[0]).any() and torch.isfinite(y[1:]).all()
        wn = w.clone()
        wn[k - 1, n - 1] = math.nan
        y, _ = ops.linear_forward(x, wn)
        assert torch.isnan(y[:, n - 1]).all() and torch.isfinite(y[:, :n - 1]).all()


def test_residual_in_place_and_repeatable():
    gen = torch.Generator(device="cuda"); gen.manual_seed(3)
    x, w, r = table(300, 1000, "bf16", gen), table(1000, 136, "bf16", gen), table(300, 136, "bf16", gen)
    y, _ = ops.linear_forward(x, w, residual=r, act="gelu")
    again, _ = ops.linear_forward(x, w, residual=r, act="gelu", out=r)
    assert again is r and torch.equal(y, r)
    first = ops.linear_backward(y, x, w)
    for a, b in zip(first, ops.linear_backward(y, x, w)):
        assert torch.equal(a, b)


def test_other_stream_and_graph():
    gen = torch.Generator(device="cuda"); gen.manual_seed(4)
    x, w, b, dy = table(100, 640, "bf16", gen), table(640, 200, "bf16", gen), table(1, 200, "bf16", gen)[0], table(100, 200, "bf16", gen)
    y, pre = ops.linear_forward(x, w, b, act="gelu", keep_pre=True)
    want = ops.linear_backward(dy, x, w, pre=pre, act="gelu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2, pre2 = ops.linear_forward(x, w, b, act="gelu", keep_pre=True)
        got = ops.linear_backward(dy, x, w, pre=pre2, act="gelu")
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(want, got))
    s.wait_stream(torch.cuda.current_stream())
    y2, pre2 = ops.linear_forward(x, w, b, act="gelu", keep_pre=True, stream=s)
    got = ops.linear_backward(dy, x, w, pre=pre2, act="gelu", stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, pre3 = ops.linear_forward(x, w, b, act="gelu", keep_pre=True)
        got = ops.linear_backward(dy, x, w, pre=pre3, act="gelu")
    for _ in range(3):
        x.copy_(table(100, 640, "bf16", gen))
        graph.replay()
        torch.cuda.synchronize()
        y, pre = ops.linear_forward(x, w, b, act="gelu", keep_pre=True)
        want = ops.linear_backward(dy, x, w, pre=pre, act="gelu")
        assert torch.equal(y, y3) and all(torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(dtype):
    """Rows that lie more than 2^32 bytes apart from the first, by their distance."""
    rows, k, n = 130, 72, 40
    ld = (1 << 32) // (rows - 2) // (2 if dtype == "bf16" else 4) // 8 * 8 + 8
    big = torch.empty(rows * ld, dtype=DT[dtype], device="cuda")
    x = big.as_strided((rows, k), (ld, 1))
    small = torch.randn(rows, k, device="cuda").to(DT[dtype])
    x.copy_(small)
    w, dy = torch.randn(k, n, device="cuda").to(DT[dtype]), torch.randn(rows, n, device="cuda").to(DT[dtype])
    assert torch.equal(ops.linear_forward(x, w)[0], ops.linear_forward(small, w)[0])
    for a, b in zip(ops.linear_backward(dy, x, w), ops.linear_backward(dy, small, w)):
        assert torch.allclose(a.float(), b.float(), rtol=2 * rounding(dtype), atol=1e-4)


# One to four rows: contractions that end inside a read, that are split, and outputs that take either number of columns for a workgroup.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1023, 31), (1, 1025, 65), (2, 2049, 10), (1, 4096, 1024), (3, 5001, 1003), (4, 4097, 4100), (1, 20011, 129), (4, 40, 16640), (2, 2050, 16390)], ids=str)
def test_few_rows(shape, dtype):
    rows, k, n = shape
    gen = torch.Generator(device="cuda"); gen.manual_seed(rows * 13 + n)
    for act, pad, shift in (("none", 0, 0), ("gelu", 3, 1)):
        x, w = table(rows, k, dtype, gen, pad, shift), table(k, n, dtype, gen, pad, shift, 1 / math.sqrt(k))
        b, r = table(1, n, dtype, gen)[0], table(rows, n, dtype, gen, pad, shift)
        y, pre = ops.linear_forward(x, w, b, residual=r, act=act, keep_pre=True)
        assert torch.equal(y, ops.linear_forward(x, w, b, residual=r, act=act)[0])
        z = x.double() @ w.double() + b.double()
        bound = (k + 8) * U * (x.double().abs() @ w.double().abs() + b.double().abs())
        close(pre, z, bound, dtype)
        close(y, act64(z, act) + r.double(), bound + U * r.double().abs(), dtype)


def test_columns_of_one_table():
    """Operands and outputs that lie side by side in the rows of one wider table share no memory."""
    gen = torch.Generator(device="cuda"); gen.manual_seed(5)
    both = torch.randn(70, 96, generator=gen, device="cuda")
    w = torch.randn(40, 56, generator=gen, device="cuda")
    want = both[:, :40].double() @ w.double()
    y, _ = ops.linear_forward(both[:, :40], w, out=both[:, 40:])
    close(y, want, 48 * U * (both[:, :40].double().abs() @ w.double().abs()), "f32")
    with pytest.raises(Exception, match="share memory"):
        ops.linear_forward(both[:, :40], w, out=both[:, 39:95])


@pytest.mark.parametrize("make,text", [
    (lambda x, w: ops.linear_forward(x.double(), w), "x must be"), (lambda x, w: ops.linear_forward(x[0], w), "x must be"), (lambda x, w: ops.linear_forward(x, w.bfloat16()), "w must be"),
    (lambda x, w: ops.linear_forward(x, w.t()), "w must be"), (lambda x, w: ops.linear_forward(x.t().contiguous().t(), w), "contiguous rows"), (lambda x, w: ops.linear_forward(x, w, w[0, :3]), "bias"),
    (lambda x, w: ops.linear_forward(x, w, w[:, 0].repeat(9)[:9]), "bias"), (lambda x, w: ops.linear_forward(x, w, residual=x), "residual must be"), (lambda x, w: ops.linear_forward(x, w, out=x), "out must be"),
    (lambda x, w: ops.linear_forward(x, w, act="tanh"), "act"), (lambda x, w: ops.linear_forward(x[:1].expand(4, 8), w), "overlap"), (lambda x, w: ops.linear_forward(x, w.cpu()), "w must be"),
    (lambda x, w: ops.linear_forward(x, w, workspace=w), "workspace"), (lambda x, w: ops.linear_backward(x, x, w), "w must be"), (lambda x, w: ops.linear_backward(x @ w, x, w, act="gelu"), "needs pre"),
    (lambda x, w: ops.linear_backward(x @ w, x[:2], w), "x must be"), (lambda x, w: ops.linear_backward(x @ w, x, w, dw=w.t()), "dw must be"), (lambda x, w: ops.linear_backward(x @ w, x, w, db=w[0, :3]), "db must be"),
    (lambda x, w: ops.cross_entropy(x, torch.zeros(4, device="cuda")), "labels"), (lambda x, w: ops.cross_entropy(x, torch.zeros(3, device="cuda", dtype=torch.int64)), "labels"),
    (lambda x, w: ops.cross_entropy(x, torch.zeros(4, dtype=torch.int64)), "labels"), (lambda x, w: ops.cross_entropy(x.half(), torch.zeros(4, device="cuda", dtype=torch.int64)), "logits must be"),
    (lambda x, w: ops.AdamW([x], [x.t()]), "grad 0"), (lambda x, w: ops.AdamW([x], [w]), "shape"), (lambda x, w: ops.AdamW([x], [x.clone()], copies=[x]), "copy 0"),
    (lambda x, w: ops.AdamW([x], [x.clone()], moments=(x, x)), "m must hold")])
def test_tensors_that_do_not_fit(make, text):
    with pytest.raises(ValueError, match=text):
        make(torch.zeros(4, 8, device="cuda"), torch.zeros(8, 5, device="cuda"))
