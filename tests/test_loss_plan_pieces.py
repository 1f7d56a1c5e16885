"""What the shapes of common_loss_shapes.py are cut into, on the host: several pieces with products in tiles of every size, with and without parts of the
contraction, and a last piece with fewer parts than the others."""
from common_loss_shapes import PIECES
from test_loss_plan import check, plan  # noqa: F401


def test_pieces_of_every_kind(plan):  # noqa: F811
    cuts = set()
    for dtype, rows, k, classes, pad in PIECES:
        f, a, dll = plan(rows, k, classes, 1 if dtype == "bf16" else 0, k + pad, classes + pad)
        check(f, a, dll)
        assert f["pieces"] > 1 and not f["kept"] and not f["left"]
        last = classes - (f["pieces"] - 1) * f["piece"]
        cuts.add((dtype, f["dx_tile"], f["dx_splits"] > 1, -(-last // f["dx_per"]) < f["dx_splits"], f["dw_splits"] > 1))
    of = lambda *at: {tuple(c[i] for i in at) for c in cuts}  # noqa: E731
    assert of(0, 1) >= {("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64)}
    assert of(0, 2) == {(t, s) for t in ("bf16", "f32") for s in (False, True)} and (256, True) in of(1, 2) and (256, False) in of(1, 2)
    assert ("bf16", True) in of(0, 3) and of(4) == {(False,), (True,)}
