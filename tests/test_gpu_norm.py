"""Layer norm and its gradients against the definitions in 64 bits.

Tolerances, with e = 2^-24 (half a step of float32) and s = (96 + width / 512) e: a lane adds up to 64 columns one after the other (wide rows: width / 1024 of them), lanes and wavefronts join in up to 32 more
additions, so a row's sum is off by s times the sum of magnitudes.
  mean: s mean|x|.                                     rstd: half of the variance's error, s + (the mean's error)^2 / variance + 2 e, and 4 e of its own operations.
  y = u w + b, u = (x - mean) rstd: u is off by |u| (rstd's error + 2 e) + rstd (the mean's error); 3 e for the product, the sum and what they are of.
  gradients, of the statistics that are handed in: u is off by 2 e |u|, g = dy w by e |g|; dx by rstd (s (mean|g| + |u| mean|g u|) + 6 e (|g| + mean|g| + |u| mean|g u|)) and e of the residual's sum;
  dw, db by (300 + rows / 16 + 4) e times the sum of magnitudes over the rows: those of a group one after the other, then 64 groups and a few hundred parts.
Outputs are rounded once more: bf16 2^-8 (eight significant bits: half a step of a value just above a power of two), float32 e."""
import pytest
import torch

from paper_2012_15469_amd import ops

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
E = 2.0 ** -24


def half_step(t):
    return 2.0 ** -8 if t.dtype == torch.bfloat16 else E


def table(gen, rows, width, dtype, pad=0, shift=0, scale=1.0, place=0.0):
    return (scale * torch.randn(rows, width + pad + shift, generator=gen, device="cuda") + place).to(DT[dtype])[:, shift:shift + width]


def near(got, want, limit, what):
    assert got.shape == want.shape
    worst = float(((got.double() - want).abs() / (limit + half_step(got) * (want.abs() + limit) + 1e-37)).max()) if got.numel() else 0.0
    assert worst <= 1.0, "%s: off by %g of its tolerance" % (what, worst)


def check_forward(x, w, b, eps, out=None):
    width = x.shape[1]
    s = (96 + width / 512) * E
    x64, w64, b64 = x.double(), 1.0 if w is None else w.double(), 0.0 if b is None else b.double()
    mean = x64.mean(1, keepdim=True)
    var = (x64 - mean).square().mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    u = (x64 - mean) * rstd
    y, m, r = ops.layer_norm_forward(x, w, b, eps=eps, keep_stats=True, out=out)
    e_mean = s * x64.abs().mean(1, keepdim=True)
    e_rstd = (s + e_mean ** 2 / (var + eps) + 2 * E) / 2 + 4 * E
    near(m, mean[:, 0], e_mean[:, 0], "mean")
    near(r, rstd[:, 0], (rstd * e_rstd)[:, 0], "rstd")
    wa = 1.0 if w is None else w64.abs()
    near(y, u * w64 + b64, wa * (u.abs() * (e_rstd + 5 * E) + rstd * e_mean) + 3 * E * (0.0 if b is None else b64.abs()), "y")
    return y, m, r


def check_backward(dy, x, m, r, w, res, **kw):
    rows, width = x.shape
    s, c = (96 + width / 512) * E, (304 + rows / 16) * E
    dy64, w64 = dy.double(), 1.0 if w is None else w.double()
    r64 = r.double()[:, None]
    u = (x.double() - m.double()[:, None]) * r64
    g = dy64 * w64
    mg, mgu, ag, agu = g.mean(1, keepdim=True), (g * u).mean(1, keepdim=True), g.abs().mean(1, keepdim=True), (g * u).abs().mean(1, keepdim=True)
    want = r64 * (g - mg - u * mgu) + (0.0 if res is None else res.double())
    e_dx = r64.abs() * (s * (ag + u.abs() * agu) + 6 * E * (g.abs() + ag + u.abs() * agu)) + E * (0.0 if res is None else want.abs() + res.double().abs())
    dx, dw, db = ops.layer_norm_backward(dy, x, m, r, w, residual=res, **kw)
    near(dx, want, e_dx, "dx")
    near(dw, (dy64 * u).sum(0), c * (dy64 * u).abs().sum(0), "dw")
    near(db, dy64.sum(0), c * dy64.abs().sum(0), "db")
    return dx, dw, db


WIDTHS = [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 63, 64, 65, 127, 129, 255, 257, 500, 513, 617, 1000, 1025, 2047, 2049, 3001, 4096, 4100, 8191, 8193, 12000, 12288, 12291, 16384, 16385, 32768, 32771, 70001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_against_definition(width, dtype):
    gen = torch.Generator(device="cuda"); gen.manual_seed(width)
    for rows, pad, shift, place, affine in ((1, 0, 0, 0.0, True), (13, 3, 1, 5.0, True), (70, 8, 0, 0.3, False)):
        x = table(gen, rows, width, dtype, pad, shift, 2.0, place)
        w, b = (table(gen, 1, width, dtype, place=1.0)[0], table(gen, 1, width, dtype)[0]) if affine else (None, None)
        _, m, r = check_forward(x, w, b, 1e-5)
        dy, res = table(gen, rows, width, dtype, pad, shift), table(gen, rows, width, dtype, 0, shift)
        check_backward(dy, x, m, r, w, res if affine else None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", [(2, 4096), (511, 1000), (513, 4096), (1030, 617), (2060, 40), (3000, 9), (5000, 3), (520, 17000), (600, 8192), (600, 9001)])
def test_many_rows(rows, width, dtype):
    """More rows than a launch has groups, so that a group takes several and the sums come in parts."""
    gen = torch.Generator(device="cuda"); gen.manual_seed(rows)
    x, w, b = table(gen, rows, width, dtype, 5), table(gen, 1, width, dtype)[0], table(gen, 1, width, dtype)[0]
    _, m, r = check_forward(x, w, b, 1e-3)
    dy, res = table(gen, rows, width, dtype, 0, 3), table(gen, rows, width, dtype)
    first = check_backward(dy, x, m, r, w, res)
    again = ops.layer_norm_backward(dy, x, m, r, w, residual=res)
    assert all(torch.equal(a, c) for a, c in zip(first, again))
    # outputs one by one
    for i, names in enumerate((("dx",), ("dw",), ("db",))):
        one = ops.layer_norm_backward(dy, x, m, r, w, residual=res, need_dx=i == 0, need_dw=i == 1, need_db=i == 2)
        assert torch.equal(one[i], first[i]) and all(one[j] is None for j in range(3) if j != i)
    assert ops.layer_norm_backward(dy, x, m, r, w, need_dx=False, need_dw=False, need_db=False) == (None, None, None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", [5, 617, 4096, 12000, 40000])
def test_in_place_and_into_wider_tables(width, dtype):
    gen = torch.Generator(device="cuda"); gen.manual_seed(7)
    x, w, b = table(gen, 300, width, dtype, 3), table(gen, 1, width, dtype)[0], table(gen, 1, width, dtype)[0]
    y, m, r = ops.layer_norm_forward(x, w, b, keep_stats=True)
    dy, res = table(gen, 300, width, dtype, 6), table(gen, 300, width, dtype, 2)
    dx, dw, db = ops.layer_norm_backward(dy, x, m, r, w, residual=res)
    for at in ("dy", "residual", "wide"):
        a, c = torch.empty(300, width + 6, dtype=x.dtype, device="cuda")[:, :width].copy_(dy), torch.empty(300, width + 2, dtype=x.dtype, device="cuda")[:, :width].copy_(res)
        wide = torch.full((302, width + 4), 7.0, dtype=x.dtype, device="cuda")
        out = {"dy": a, "residual": c, "wide": wide[1:301, 2:2 + width]}[at]
        dx2, dw2, db2 = ops.layer_norm_backward(a, x, m, r, w, residual=c, dx=out)
        assert dx2 is out and torch.equal(dx2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)
        if at == "wide":
            wide[1:301, 2:2 + width] = 7.0
            assert bool((wide == 7.0).all())
    z = torch.empty(300, width + 3, dtype=x.dtype, device="cuda")[:, :width].copy_(x)
    assert ops.layer_norm_forward(z, w, b, out=z)[0] is z and torch.equal(z, y)


def test_rows_where_it_can_go_wrong():
    """Constant rows, rows whose squares leave float32 only in the sum, one large value, infinities and NaN: each row by itself."""
    for width in (8, 300, 5000, 40000):
        x = torch.randn(9, width, device="cuda")
        x[0] = 3.0
        x[1] = 0.0
        x[2] = 1e4 + x[2] * 1e-2
        x[3] *= 1e-15
        x[4, 0] = 1e15
        x[5, 1] = float("inf")
        x[6, 1] = float("nan")
        x[7, 1] = -float("inf")
        y, m, r = ops.layer_norm_forward(x, keep_stats=True)
        assert not y[0:2].any() and bool((m[0:2] == torch.tensor([3.0, 0.0], device="cuda")).all()) and bool(((r[0:2] * 1e-5 ** 0.5 - 1).abs() < 1e-6).all())
        check_forward(x[2:5], None, None, 1e-5)
        check_forward(x[8:], None, None, 1e-5)
        assert bool(torch.isnan(y[5:8]).any(1).all()) and bool(torch.isfinite(y[8]).all())
        dx, dw, db = ops.layer_norm_backward(torch.randn_like(x[[0, 1, 8]]), x[[0, 1, 8]].contiguous(), m[[0, 1, 8]], r[[0, 1, 8]])
        assert bool(torch.isfinite(dx).all())


def test_no_rows():
    x = torch.empty(0, 33, device="cuda")
    y, m, r = ops.layer_norm_forward(x, keep_stats=True)
    assert y.shape == (0, 33) and m.shape == r.shape == (0,)
    dx, dw, db = ops.layer_norm_backward(x, x, m, r)
    assert dx.shape == (0, 33) and dw.shape == db.shape == (33,) and not dw.any() and not db.any()


def test_gradient_against_differences():
    """Central differences of the definition in 64 bits (step 1e-5: their error is below 1e-8)."""
    gen = torch.Generator(device="cuda"); gen.manual_seed(3)
    x, w, b, dy = table(gen, 3, 11, "f32"), table(gen, 1, 11, "f32")[0], table(gen, 1, 11, "f32")[0], table(gen, 3, 11, "f32")

    def value(x, w, b):
        c = x - x.mean(1, keepdim=True)
        return ((c / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-5) * w + b) * dy.double()).sum()

    _, m, r = ops.layer_norm_forward(x, w, b, keep_stats=True)
    got = ops.layer_norm_backward(dy, x, m, r, w)
    leaves = [t.double() for t in (x, w, b)]
    for which, leaf in enumerate(leaves):
        flat = leaf.view(-1)
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + 1e-5
            hi = float(value(*leaves))
            flat[i] = old - 1e-5
            lo = float(value(*leaves))
            flat[i] = old
            assert abs(float(got[which].view(-1)[i]) - (hi - lo) / 2e-5) < 1e-5


def test_graph_replays_and_another_stream():
    x, w, b, dy = torch.randn(700, 1000, device="cuda").to(torch.bfloat16), torch.randn(1000, device="cuda").to(torch.bfloat16), torch.randn(1000, device="cuda").to(torch.bfloat16), torch.randn(700, 1000, device="cuda").to(torch.bfloat16)

    def both(**kw):
        y, m, r = ops.layer_norm_forward(x, w, b, keep_stats=True, **kw)
        return (y, m, r, *ops.layer_norm_backward(dy, x, m, r, w, **kw))

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        x.copy_(torch.randn(700, 1000, device="cuda"))
        dy.copy_(torch.randn(700, 1000, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, both()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    there = both(stream=side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, there))


def test_rows_far_apart():
    """Rows more than 4 GB apart."""
    apart = (1 << 31) + 64
    base = torch.empty(2 * apart + 1000, dtype=torch.bfloat16, device="cuda")
    x = base.as_strided((3, 1000), (apart, 1))
    x.copy_(torch.randn(3, 1000, device="cuda"))
    near_x = x.contiguous()
    y, m, r = ops.layer_norm_forward(near_x, keep_stats=True)
    y2, m2, r2 = ops.layer_norm_forward(x, keep_stats=True, out=x)
    assert torch.equal(y, y2) and torch.equal(m, m2) and torch.equal(r, r2)
    dx, dw, db = ops.layer_norm_backward(y, near_x, m, r)
    dx2, dw2, db2 = ops.layer_norm_backward(x, near_x, m, r, dx=x)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("kw,text", [
    (dict(weight=torch.zeros(3)), "weight must be a contiguous"), (dict(bias=torch.zeros(8, dtype=torch.float64)), "bias must be a contiguous"), (dict(out=torch.zeros(4, 8)), "out must be Float on cuda"),
    (dict(mean=torch.zeros(3)), "mean must be a contiguous Float")])
def test_refusals(kw, text):
    x = torch.zeros(4, 8, device="cuda")
    with pytest.raises(ValueError, match=text):
        ops.layer_norm_forward(x, **kw)
    with pytest.raises(ValueError, match="contiguous rows"):
        ops.layer_norm_forward(torch.zeros(8, 4, device="cuda").t())
    with pytest.raises(ValueError, match="rstd must be"):
        ops.layer_norm_backward(x, x, torch.zeros(4, device="cuda"), torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError, match="x must be"):
        ops.layer_norm_backward(x, x[:, :4], torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"))
