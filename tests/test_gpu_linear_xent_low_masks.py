"""The loss of a last layer with smoothed labels and a bias of the type's lowest value at most of its classes: such a class is not ruled out, so the loss is
smoothing times the mean distance of the logits from the label's, some 3e37, which float32 has, although two of its terms together are more than float32
has.

Tolerances, with e = 2^-24: the loss is a sum of one sign, but for the ordinary logits, which are less than a step of it; each of its terms is off by 4 e
relative (the logit, the difference, the factor, the sum it enters), an addition by e, of which there are 64 one after the other in a strip of columns, up
to classes / 32 strips, and 32 in the joins, and the last operations take 8: (classes / 32 + 108) e in all.  Probabilities and gradients are those of a mask
at -120, whose exponential, 8e-53, is as good as zero: their tolerances are the ones of the formulas there."""
import pytest
import torch

from paper_2012_15469_amd import ops
from test_gpu_linear_xent import DT, E, definition, near, problem

pytestmark = pytest.mark.gpu

# rows, in, classes: logits that are kept (of one and of several lanes' pieces), that the statistics leave behind, that are formed again, in tiles of every size, one piece and several
SHAPES = [(12, 64, 5), (12, 64, 200), (12, 64, 3000), (300, 40, 1001), (2500, 24, 900), (40, 33, 16001), (6, 64, 20000), (300, 50, 30001), (4100, 64, 20008),
          (20000, 16, 3000), (64, 72, 65536), (1, 40, 40000)]


def lowest(rows, k, classes, dtype, share):
    """All classes at the lowest value but a few, a label's among them; a share of them ruled out besides."""
    x, w, labels, b = problem(rows, k, classes, dtype, 21, ignored=0.1 if rows > 1 else 0.0)
    gen = torch.Generator(device="cuda"); gen.manual_seed(classes)
    ordinary = torch.rand(classes, generator=gen, device="cuda") < 0.1
    ordinary[1] = True
    out = torch.rand(classes, generator=gen, device="cuda") < share
    out[1] = out[0] = False
    ordinary[0] = False
    b = torch.where(ordinary, b, torch.tensor(torch.finfo(b.dtype).min, dtype=b.dtype, device="cuda")).masked_fill(out, -float("inf"))
    allowed = torch.nonzero(ordinary & ~out)[:, 0]
    labels = torch.where(labels < 0, labels, allowed[labels.clamp(min=0) % allowed.numel()])
    return x, w, labels, b


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,classes", SHAPES)
def test_lowest_values(rows, k, classes, dtype):
    for share in (0.0, 0.3):
        x, w, labels, b = lowest(rows, k, classes, dtype, share)
        want = definition(x, w, labels, b, 0.1, -100, 1.0)[0]
        used = labels != -100
        assert bool((want[used] > 1e36).all()) and bool((want < 3e38).all())
        rel = (classes / 32 + 108) * E
        tame = torch.where(b == torch.finfo(b.dtype).min, torch.tensor(-120.0, dtype=b.dtype, device="cuda"), b)
        _, g, e_g, _, count = definition(x, w, labels, tame, 0.1, -100, 1.0)
        e_s = e_g + (2.0 ** -8 * (g.abs() + e_g) if dtype == "bf16" else 0.0)
        x64, w64 = torch.where(used[:, None], x.double(), 0.0), w.double()
        for grads in (False, True):
            mean, loss, dx, dw, db = ops.linear_cross_entropy(x, w, labels, b, smoothing=0.1, need_dx=grads, need_dw=grads, need_db=grads)
            near(loss, want, rel * want.abs(), "loss")
            near(mean, want.sum() / count, rel * want.abs().sum() / count, "mean")
        near(dx, g @ w64.t(), e_s @ w64.abs().t() + (classes + 2) * E * (g.abs() @ w64.abs().t()), "dx")
        near(dw, x64.t() @ g, x64.abs().t() @ e_s + (rows + 2) * E * (x64.abs().t() @ g.abs()), "dw")
        near(db, g.sum(0), e_g.sum(0) + (rows + 2) * E * g.abs().sum(0), "db")
        if rows * classes < 1 << 24:          # as cross_entropy has it, of this library's own logits
            z, _ = ops.linear_forward(x, w, b)
            there = ops.cross_entropy(z, labels, smoothing=0.1)[1].double()
            near(loss, there, 2 * rel * want.abs(), "loss of the two operators apart")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(12, 200), (12, 3000), (6, 20000), (2500, 900), (1, 1)])
def test_nothing_but_lowest_values(rows, classes, dtype):
    """Every class at the lowest value: logits as far from each other as the products are, none of which the type's lowest value shows; the loss is that of
    even classes."""
    x, w, labels, _ = problem(rows, 30, classes, dtype, 22)
    b = torch.full((classes,), torch.finfo(DT[dtype]).min, dtype=DT[dtype], device="cuda")
    for grads in (False, True):
        loss = ops.linear_cross_entropy(x, w, labels, b, smoothing=0.1, need_dx=grads, need_dw=grads, need_db=grads)[1]
        assert float((loss.double() - torch.tensor(float(classes), dtype=torch.float64).log().item()).abs().max()) <= (classes / 32 + 108) * E * 20
